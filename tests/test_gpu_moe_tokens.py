"""ccl_moe_tokens against the layer in 64 bits: one token to the most, one expert to 512, odd widths, strips, ties and NaN.

Bounds (u, e as in ffn_reference.py): logits, gate and up are fp32 sums of exact products; in whatever order, a sum of K terms is off
by at most (K/8 + 64) e of the sum of the terms' magnitudes here (8-wide partial sums, 16-deep tensor-core steps, then trees).  The weights
follow the logits' error; h is rounded to bf16 once; Y is rounded once."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import E, U, act, assert_within

pytestmark = pytest.mark.gpu


def make(T, E_, H, I, seed, std=0.05):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, s=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * s).to(torch.bfloat16)

    return normal(T, H), normal(E_, H, s=std), normal(E_, 2 * I, H, s=std), normal(E_, H, I, s=std), normal(T, H)


def reference(x, wr, wgu, wd, res, topk, norm, strips, ids):
    """The layer in 64 bits with the given choice of experts -> (Y, bound of the error, weights, bound of theirs)."""
    T, H = x.shape
    I = wd.shape[2]
    x, wr = x.double(), wr.double()
    logits = x @ wr.t()
    l_err = (H / 8 + 64) * E * (x.abs() @ wr.abs().t())
    l, le = logits.gather(1, ids), l_err.gather(1, ids)
    p = torch.exp(l - logits.max(1, keepdim=True).values)
    full = torch.exp(logits - logits.max(1, keepdim=True).values).sum(1, keepdim=True)
    w = p / (p.sum(1, keepdim=True) if norm else full)
    w_err = w * (2 * l_err.max(1, keepdim=True).values + 600 * E)           # softmax moves by at most twice the logits' error; sums of up to 512 terms
    y = res.double() if res is not None else torch.zeros(T, H, dtype=torch.float64, device="cuda")
    err = E * y.abs()
    half = I // strips
    for e in ids.unique().tolist():
        t, k = (ids == e).nonzero(as_tuple=True)
        g = wgu[e].double().reshape(strips, 2, half, H)
        gate_w, up_w = g[:, 0].reshape(I, H), g[:, 1].reshape(I, H)
        gate, up = x[t] @ gate_w.t(), x[t] @ up_w.t()
        ge, ue = (H / 8 + 64) * E * (x[t].abs() @ gate_w.abs().t()), (H / 8 + 64) * E * (x[t].abs() @ up_w.abs().t())
        h = act(gate, "silu") * up
        he = (1.13 * ge + 2.0 ** -20 * (1 + gate.abs())) * (up.abs() + ue) + act(gate, "silu").abs() * ue
        he = he + U * (h.abs() + he)
        d = wd[e].double()
        o = h @ d.t()
        oe = he @ d.abs().t() + (I / 8 + 64) * E * ((h.abs() + he) @ d.abs().t())
        wk, wke = w[t, k][:, None], w_err[t, k][:, None]
        y[t] += wk * o
        err[t] += wk * oe + wke * (o.abs() + oe) + 64 * E * (wk * o).abs()
    return y, err + U * (y.abs() + err), w, w_err


def run(x, wr, wgu, wd, res, topk, norm, strips=1, ws=None, **strides):
    T, H = x.shape
    E_, _, I = wd.shape if wd.dim() == 3 else (wr.shape[0], 0, strides.pop("I"))
    d = ccl.MoeDesc(T, E_, topk, H, I, norm_topk=int(norm), gu_strips=strips, **strides)
    need = ccl.ccl_moe_tokens_workspace(d)
    if ws is None:
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")             # NaN wherever it is read before it is written
    y = torch.full((T * H + 64,), 0x7FC0, dtype=torch.int16, device="cuda")
    ids = torch.full((T * topk + 16,), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T * topk + 16,), -7.0, dtype=torch.float32, device="cuda")
    ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws[:need], residual=res, ids=ids, weights=w)
    st, detail = ccl.ccl_gemm_status()
    assert st == ccl.OK, detail
    assert (y[T * H:] == 0x7FC0).all() and (ids[T * topk:] == -7).all() and (w[T * topk:] == -7.0).all() and (ws[need:] == 0xFF).all()
    return y[:T * H].view(torch.bfloat16).view(T, H), ids[:T * topk].view(T, topk).long(), w[:T * topk].view(T, topk)


def check(T, E_, topk, H, I, norm=True, residual=True, strips=1, seed=0):
    x, wr, wgu, wd, res = make(T, E_, H, I, seed)
    res = res if residual else None
    y, ids, w = run(x, wr, wgu, wd, res, topk, norm, strips)
    logits = x.double() @ wr.double().t()
    l_err = (H / 8 + 64) * E * (x.double().abs() @ wr.double().abs().t())
    # the choice: distinct experts, best first, none left out that is better by more than the logits' error
    assert (ids >= 0).all() and (ids < E_).all() and all(len(set(r)) == topk for r in ids.tolist())
    chosen, ce = logits.gather(1, ids), l_err.gather(1, ids)
    assert (chosen[:, 1:] - ce[:, 1:] <= chosen[:, :-1] + ce[:, :-1]).all()
    rest = logits.clone().scatter_(1, ids, float("-inf"))
    assert (rest - l_err <= (chosen[:, -1:] + ce[:, -1:])).all()
    want, bound, ww, we = reference(x, wr, wgu, wd, res, topk, norm, strips, ids)
    assert_within(w, ww, we, "weights")
    assert_within(y, want, bound, "Y")


CASES = [
    # T, E, topk, H, I
    (1, 1, 1, 8, 8), (1, 8, 2, 512, 256), (1, 128, 8, 2048, 768), (2, 16, 4, 136, 72), (3, 60, 4, 1544, 712), (5, 512, 16, 264, 40), (7, 60, 4, 1544, 712),
    (8, 32, 8, 1024, 520), (9, 32, 8, 1024, 520), (16, 64, 6, 2048, 768), (17, 8, 2, 520, 1032), (33, 8, 8, 264, 136), (64, 128, 8, 512, 256), (64, 8, 2, 1024, 384),
    (64, 4, 4, 2048, 128), (64, 512, 16, 256, 64), (40, 1, 1, 640, 200), (4, 16, 2, 4104, 264), (20, 16, 2, 8192, 72), (1, 4, 2, 2400, 1536), (64, 60, 16, 2376, 520),
]


@pytest.mark.parametrize("T,E_,topk,H,I", CASES)
def test_layer(T, E_, topk, H, I):
    check(T, E_, topk, H, I, norm=True, residual=True, seed=T)
    check(T, E_, topk, H, I, norm=False, residual=False, seed=T + 100)


@pytest.mark.parametrize("strips", [2, 4])
def test_gate_up_in_strips(strips):
    check(6, 16, 4, 512, 768, strips=strips)
    check(40, 16, 4, 512, 768, strips=strips)


def test_expert_strides_and_offsets_past_32_bits():
    T, E_, topk, H, I = 3, 5, 3, 512, 128
    x, wr, wgu, wd, res = make(T, E_, H, I, 5)
    far_gu, far_d = (1 << 30) + 16, (1 << 30) - 4096                        # the last expert starts past 4 GB
    big_gu = torch.zeros((far_gu * (E_ - 1) + 4 * I * H) // 2, dtype=torch.bfloat16, device="cuda")
    big_d = torch.zeros((far_d * (E_ - 1) + 2 * I * H) // 2, dtype=torch.bfloat16, device="cuda")
    for e in range(E_):
        big_gu[far_gu // 2 * e:][:2 * I * H] = wgu[e].reshape(-1)
        big_d[far_d // 2 * e:][:I * H] = wd[e].reshape(-1)
    a = run(x, wr, wgu, wd, res, topk, True)
    b = run(x, wr, big_gu, big_d, res, topk, True, I=I, gu_stride_bytes=far_gu, d_stride_bytes=far_d)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_equal_logits_go_to_the_lowest_expert():
    for T, E_, topk in ((1, 128, 8), (12, 60, 5), (3, 512, 16)):
        x, wr, wgu, wd, res = make(T, E_, 256, 64, 1)
        wr[:] = wr[3]                                                       # every expert alike
        _, ids, w = run(x, wr, wgu, wd, res, topk, True)
        assert (ids == torch.arange(topk, device="cuda")).all()
        assert_within(w, torch.full_like(w, 1 / topk).double(), torch.tensor(32 * E, device="cuda"), "weights")


def test_nan_and_infinity_stay_with_their_token():
    T, E_, topk, H, I = 12, 16, 3, 256, 64
    x, wr, wgu, wd, res = make(T, E_, H, I, 2)
    y0, ids0, w0 = run(x, wr, wgu, wd, res, topk, True)
    x[4, 17] = float("nan")
    x[7, 3] = float("inf")
    y, ids, w = run(x, wr, wgu, wd, res, topk, True)
    keep = [t for t in range(T) if t not in (4, 7)]
    assert torch.isnan(y[4]).all() and torch.isnan(w[4]).all() and torch.isnan(y[7]).all()
    assert torch.equal(ids[keep], ids0[keep]) and torch.equal(w[keep], w0[keep]) and torch.equal(y[keep], y0[keep])
    assert all(len(set(r)) == topk and 0 <= min(r) and max(r) < E_ for r in ids.tolist())
    # an expert whose router row is NaN is never chosen before a number
    x, wr, wgu, wd, res = make(T, E_, H, I, 2)
    wr[5] = float("nan")
    _, ids, w = run(x, wr, wgu, wd, res, topk, False)
    assert not (ids == 5).any() and torch.isnan(w).all()


def test_residual_in_place_and_repeated_runs():
    for T in (1, 8, 20):
        x, wr, wgu, wd, res = make(T, 32, 1024, 256, 3)
        y0, ids0, w0 = run(x, wr, wgu, wd, res, 4, True)
        d = ccl.MoeDesc(T, 32, 4, 1024, 256)
        ws = torch.zeros(ccl.ccl_moe_tokens_workspace(d), dtype=torch.uint8, device="cuda")
        for _ in range(20):                                                 # back to back, one workspace, no synchronisation in between
            y = res.clone()
            ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws, residual=y)
            assert torch.equal(y, y0)
        assert ccl.ccl_gemm_status()[0] == ccl.OK


def test_graph_replay_and_another_stream():
    x, wr, wgu, wd, res = make(4, 32, 1024, 256, 4)
    y0, _, _ = run(x, wr, wgu, wd, res, 4, True)
    d = ccl.MoeDesc(4, 32, 4, 1024, 256)
    ws = torch.full((ccl.ccl_moe_tokens_workspace(d),), 0xA5, dtype=torch.uint8, device="cuda")
    y = torch.zeros(4, 1024, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws, residual=res)
    side.synchronize()
    assert torch.equal(y, y0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws, residual=res)
        ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws, residual=res)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y0)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
