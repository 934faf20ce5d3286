"""ccl_linear_xent and ccl_linear_xent_grad against their formulas in 64 bits: vocabularies and token counts that no tile divides, both storages of the
weight, ignored rows, several pieces.

Bounds (u = 2^-8, e = 2^-23; ffn_reference.py's product bound b(z) for a logit):
  lse    a change of the logits moves it by their mean under p: sum p b(z); an exponential is off by 2^-21 and by the rounding of z log2 e, e |z|;
         the sums are at most 128 + V/128 additions deep: 2^-20 + (128 + V/128) e + 2 e max|z| + e |lse|
  loss   those of lse and of the target's logit
  dz     |dloss| p (b(z) + 2^-20 + 2 e |z| + 2 e |lse|) + 2 e |dz|, then u of it (bf16)
  dX, dW dz's bound through the product, the product's own bound, then u
  Below 2^-126, the least normal number of fp32 and of bf16, exponentials, their products with dloss and results may be flushed to zero:
  2^-126 (1 + |dloss|) for dz, 2^-126 more for an output.
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import E, U, assert_within, product_bound
from test_gpu_gemm_epilogue import forced, workspace

pytestmark = pytest.mark.gpu

IGNORE = -100
TINY = 2.0 ** -126


class Problem:
    """Inputs, and everything in 64 bits."""

    def __init__(self, T, V, H, P=1, trans=True, align=0, ignored=0.2, seed=0, std=0.05, lean=6.0, ignore=IGNORE):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda")              # noqa: E731
        self.T, self.V, self.H = T, V, H
        w = (normal(V, H) * std).to(torch.bfloat16)
        self.targets = torch.randint(0, V, (T,), generator=g, device="cuda")
        x = normal(T, H)
        x += w[self.targets].float() * (lean * torch.rand(T, 1, generator=g, device="cuda") / (std * std * H))
        self.x = x.to(torch.bfloat16)
        self.live = torch.rand(T, generator=g, device="cuda") >= ignored
        self.tg = torch.where(self.live, self.targets, ignore).to(torch.int32)
        self.m = ccl.Mat(V, H, 2) if trans else ccl.Mat(H, V, 2, P, ccl.PART_COLS if P > 1 else ccl.PART_NONE, ccl.CCL if P > 1 else ccl.ROWMAJOR, align)
        self.d = ccl.XentDesc(T, V, H, self.m, w_trans=int(trans), ignore_index=ignore)
        self.trans = trans
        if trans:
            self.w = w
        else:
            self.w = torch.zeros(ccl.ccl_buffer_bytes(self.m) // 2, dtype=torch.bfloat16, device="cuda")
            ccl.ccl_repack(self.m, w.t().contiguous(), self.w)
        self.w64, self.x64 = w.double(), self.x.double()
        self.z = self.x64 @ self.w64.t()
        self.zb = product_bound(self.x64, self.w64.t())
        self.lse = torch.logsumexp(self.z, 1)
        self.p = (self.z - self.lse[:, None]).exp()
        self.dloss = (normal(T) / T).float()

    def forward(self, want=("loss", "lse")):
        T = self.T
        loss = torch.full((T + 8,), 7.0, device="cuda") if "loss" in want else None
        lse = torch.full((T + 8,), 7.0, device="cuda") if "lse" in want else None
        ccl.ccl_linear_xent(self.d, self.x, self.w, self.tg, loss, lse, workspace(ccl.ccl_linear_xent_workspace(self.d)))
        return loss, lse

    def check_forward(self, status=True, **kw):
        loss, lse = self.forward(**kw)
        T, V = self.T, self.V
        lse_err = (self.p * self.zb).sum(1) + 2.0 ** -20 + (128 + V / 128) * E + 2 * E * self.z.abs().amax(1) + E * self.lse.abs()
        if lse is not None:
            assert_within(lse[:T], self.lse, lse_err, "lse")
            assert (lse[T:] == 7.0).all()
        if loss is not None:
            at = self.z.gather(1, self.targets[:, None])[:, 0]
            at_err = self.zb.gather(1, self.targets[:, None])[:, 0]
            want = torch.where(self.live, self.lse - at, torch.zeros_like(at))
            assert_within(loss[:T], want, torch.where(self.live, lse_err + at_err + E * (at.abs() + want.abs()), torch.zeros_like(at)), "loss")
            assert (loss[T:] == 7.0).all()
        if status:
            assert ccl.ccl_gemm_status()[0] == ccl.OK

    def grad(self, dx=True, dw=True):
        guard = 64
        dX = torch.full((self.T * self.H + guard,), 7.0, dtype=torch.bfloat16, device="cuda") if dx else None
        n = ccl.ccl_buffer_bytes(self.m) // 2
        dW = torch.full((n + guard,), 7.0, dtype=torch.bfloat16, device="cuda") if dw else None
        ccl.ccl_linear_xent_grad(self.d, self.x, self.w, self.tg, self.lse.float(), self.dloss, dX, dW, workspace(ccl.ccl_linear_xent_grad_workspace(self.d)))
        if dx:
            assert (dX[self.T * self.H:] == 7.0).all(), "dX: wrote past the end"
        if dw:
            assert (dW[n:] == 7.0).all(), "dW: wrote past the end"
        return dX, dW

    def check_grad(self, **kw):
        dX, dW = self.grad(**kw)
        dl = (self.dloss.double() * self.live)[:, None]
        hot = torch.zeros_like(self.p).scatter_(1, self.targets[:, None], 1.0)
        dz = dl * (self.p - hot)
        err = dl.abs() * self.p * (self.zb + 2.0 ** -20 + 2 * E * self.z.abs() + 2 * E * self.lse.abs()[:, None]) + 2 * E * dz.abs()
        err = err + U * (dz.abs() + err) + TINY * (1 + dl.abs())
        if dX is not None:
            want = dz @ self.w64
            e = err @ self.w64.abs() + product_bound(dz.abs() + err, self.w64)
            assert_within(dX[:self.T * self.H].view(self.T, self.H), want, e + U * (want.abs() + e) + TINY, "dX")
        if dW is not None:
            want = dz.t() @ self.x64
            e = err.t() @ self.x64.abs() + product_bound((dz.abs() + err).t(), self.x64)
            if self.trans:
                got = dW[:self.V * self.H].view(self.V, self.H)
            else:
                got = torch.empty(self.H, self.V, dtype=torch.bfloat16, device="cuda")
                ccl.ccl_repack(self.m, dW, got, 1)
                got = got.t()
            assert_within(got, want, e + U * (want.abs() + e) + TINY, "dW")
        assert ccl.ccl_gemm_status()[0] == ccl.OK


SIZES = [(1, 1, 8), (1, 2, 16), (3, 10, 24), (7, 65, 64), (1, 5000, 2048), (19, 1001, 72), (33, 8, 520), (130, 777, 200), (128, 256, 64), (129, 257, 64), (64, 4096, 128),
         (257, 2503, 200), (300, 640, 1544), (5, 50001, 64), (1000, 3001, 96), (2, 1000, 8192)]


@pytest.mark.parametrize("T,V,H", SIZES)
def test_row_major(T, V, H):
    p = Problem(T, V, H, seed=T + V)
    p.check_forward()
    p.check_grad()


@pytest.mark.parametrize("ctas,bn", [(1, 128), (1, 256), (2, 128), (2, 256)])
@pytest.mark.parametrize("T,V,H", [(300, 3001, 136), (300, 3001, 1600), (40, 20011, 64)])
def test_every_tile(T, V, H, ctas, bn):
    with forced(ctas=ctas, bn=bn):
        p = Problem(T, V, H, seed=5)
        p.check_forward()
        p.check_grad()


STRIPS = [(40, 1024, 64, 4, 0), (130, 3 * 200, 72, 3, 0), (65, 2 * 1000, 136, 2, 4096), (300, 4 * 648, 520, 4, 0), (1, 4096, 256, 4, 0), (257, 8 * 64, 64, 8, 256), (50, 512, 128, 1, 0),
          (9, 1048, 40, 1, 0)]


@pytest.mark.parametrize("T,V,H,P,align", STRIPS)
def test_strips(T, V, H, P, align):
    # (strips that are not a multiple of 64 columns go one by one: several pieces, dX summed over them)
    p = Problem(T, V, H, P, trans=False, align=align, seed=T)
    p.check_forward()
    p.check_grad()


def test_strips_with_few_tokens_split_the_sum_of_dx():
    # 16 tokens, 5 pieces of 6008 classes: two tiles of dX, whose K the plan splits
    p = Problem(16, 5 * 6008, 256, 5, trans=False, seed=3)
    sums = ccl.ccl_linear_xent_grad_workspace(p.d) - 16 * 6008 * 2
    assert sums >= 2 * 16 * 256 * 4
    p.check_grad()


def test_several_pieces_of_a_row_major_weight():
    p = Problem(4100, 66003, 64, seed=8)                        # dz of all classes would take 541 MB
    assert ccl.ccl_linear_xent_grad_workspace(p.d) < 4100 * 66003 * 2
    p.check_forward()
    p.check_grad()


def test_wanted_outputs_only():
    p = Problem(70, 900, 64, seed=2)
    p.check_forward(want=("loss",))
    p.check_forward(want=("lse",))
    p.check_grad(dw=False)
    p.check_grad(dx=False)


def test_ignored_rows():
    p = Problem(50, 700, 64, ignored=1.0, seed=4)               # every row
    p.check_forward()
    dX, dW = p.grad()
    assert (dX[:-64] == 0).all() and (dW[:-64] == 0).all()
    p = Problem(50, 700, 64, ignored=0.3, seed=4, ignore=5)     # an index that is a class
    p.targets[p.targets == 5] = 6
    p.tg = torch.where(p.live, p.targets, 5).to(torch.int32)
    p.check_forward()
    p.check_grad()


def test_targets_outside_are_ignored_and_reported():
    p = Problem(40, 600, 64, ignored=0.0, seed=6)
    p.tg[3], p.tg[30], p.tg[31] = 600, -1, 2 ** 31 - 1
    p.live[3] = p.live[30] = p.live[31] = False
    p.check_forward(status=False)
    assert ccl.ccl_gemm_status() == (ccl.ERR_SHAPE, 10)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
    p.check_grad()


def test_extreme_logits():
    # logits of thousands: their exponentials only exist about the largest
    p = Problem(30, 500, 64, std=4.0, seed=7, lean=20000.0)
    assert p.z.abs().max() > 5000
    p.check_forward()
    p.check_grad()
    p = Problem(30, 500, 64, std=0.0 + 1e-30, seed=7, lean=0.0)  # all logits alike
    p.check_forward()


def test_non_finite_rows_stay_by_themselves():
    p = Problem(60, 500, 64, ignored=0.0, seed=9)
    p.x[7, 3] = float("nan")
    p.x[8, 3] = float("inf")
    loss, lse = p.forward()
    bad = torch.zeros(60, dtype=torch.bool, device="cuda")
    bad[7] = bad[8] = True
    assert not torch.isfinite(lse[:60][bad]).any() and torch.isfinite(lse[:60][~bad]).all()
    want = torch.logsumexp(p.z, 1)
    assert (lse[:60][~bad].double() - want[~bad]).abs().max() < 1e-4


def test_same_bits_on_every_run_on_streams_and_in_a_graph():
    p = Problem(500, 3000, 256, seed=10)
    want = [t.clone() for t in (*p.forward(), *p.grad())]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = [*p.forward(), *p.grad()]
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    loss, lse = torch.empty(500, device="cuda"), torch.empty(500, device="cuda")
    dX, dW = torch.empty_like(p.x), torch.empty_like(p.w)
    ws, gs = workspace(ccl.ccl_linear_xent_workspace(p.d)), workspace(ccl.ccl_linear_xent_grad_workspace(p.d))
    exact = p.lse.float()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ccl.ccl_linear_xent(p.d, p.x, p.w, p.tg, loss, lse, ws)
        ccl.ccl_linear_xent_grad(p.d, p.x, p.w, p.tg, exact, p.dloss, dX, dW, gs)
    for _ in range(2):
        for t in (loss, lse, dX, dW):
            t.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (loss, lse, dX.view(-1), dW.view(-1))):
            assert torch.equal(a[:b.numel()], b)


def test_against_differences():
    T, V, H, step = 12, 300, 64, 1e-4
    p = Problem(T, V, H, ignored=0.2, seed=11)
    dX, dW = (t[:-64].double() for t in p.grad())
    g = torch.Generator(device="cuda").manual_seed(1)
    D, DW = torch.randn(T, H, generator=g, device="cuda", dtype=torch.float64), torch.randn(V, H, generator=g, device="cuda", dtype=torch.float64)

    def value(x, w):
        z = x @ w.t()
        return ((torch.logsumexp(z, 1) - z.gather(1, p.targets[:, None])[:, 0]) * p.dloss.double() * p.live).sum()

    for got, d, along in ((dX.view(T, H), D, (value(p.x64 + step * D, p.w64) - value(p.x64 - step * D, p.w64)) / (2 * step)),
                          (dW.view(V, H), DW, (value(p.x64, p.w64 + step * DW) - value(p.x64, p.w64 - step * DW)) / (2 * step))):
        # u of every entry for its own rounding and as much again for dz's, summed; the difference's own error is of the order of step^2
        assert abs((got * d).sum() - along) <= 3 * U * (got * d).abs().sum() + 1e-4 * along.abs() + 1e-6


def test_offsets_past_32_bits():
    T, V, H = 8, 140001, 16384                                  # 2.3e9 elements of W: the last classes lie behind 4 GB
    w = torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    w[-T:] = (x.float() * (8.0 / H)).to(torch.bfloat16)          # class V - T + t has a logit of about 8 for token t, all others about 0
    targets = torch.arange(V - T, V, device="cuda", dtype=torch.int32)
    d = ccl.XentDesc(T, V, H)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ccl.ccl_linear_xent(d, x, w, targets, loss, lse, workspace(ccl.ccl_linear_xent_workspace(d)))
    z = x.double() @ w[-T:].double().t()
    want = torch.log(z.exp().sum(1) + (V - T))
    assert (lse.double() - want).abs().max() < 1e-4 and (loss.double() - (want - z.diagonal())).abs().max() < 1e-3
    dloss = torch.ones(T, device="cuda")
    dw = torch.full_like(w, 3.0)
    dx = torch.empty_like(x)
    ccl.ccl_linear_xent_grad(d, x, w, targets, want.float(), dloss, dx, dw, workspace(ccl.ccl_linear_xent_grad_workspace(d)))
    dz = (z - want[:, None]).exp() - torch.eye(T, device="cuda", dtype=torch.float64)
    assert ((dw[-T:].double() - dz.t() @ x.double()).abs() <= 3 * U * (dz.abs().t() @ x.double().abs()) + 1e-3).all()
    assert ((dx.double() - dz @ w[-T:].double()).abs() <= 3 * U * (dz.abs() @ w[-T:].double().abs()) + 1e-6).all()
    rest = (-want[:, None]).exp().t() @ x.double()               # every other class
    assert ((dw[:5].double() - rest).abs() <= 3 * U * ((-want[:, None]).exp().t() @ x.double().abs())).all()
