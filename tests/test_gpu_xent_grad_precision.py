"""The gradients of ccl_linear_xent with up to 16 tokens, whose dz have few others to average their roundings with and are kept in twice as many bits.

Bounds (u = 2^-8, the half step of bf16; e = 2^-23), as in test_gpu_linear_xent.py but for dz: kept as a bf16 and what is left of it as another, it is off by
u^2 of itself.  dX and dW: dz's bound through the product, the product's own, then u of the value for its rounding.
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import E, U, assert_within, product_bound
from test_gpu_gemm_epilogue import forced
from test_gpu_linear_xent import TINY, Problem

pytestmark = pytest.mark.gpu


def check(p):
    dX, dW = p.grad()
    dl = (p.dloss.double() * p.live)[:, None]
    hot = torch.zeros_like(p.p).scatter_(1, p.targets[:, None], 1.0)
    q = torch.exp(p.z - p.lse.float().double()[:, None])        # (from the lse that the call gets)
    dz = dl * (q - hot)
    err = dl.abs() * q * (p.zb + 2.0 ** -20 + 2 * E * p.z.abs() + 2 * E * p.lse.abs()[:, None]) + 2 * E * (dz.abs() + dl.abs() * hot)
    err = err + U * U * (dz.abs() + err) + TINY * (1 + dl.abs())
    pairs = [(dX[:p.T * p.H].view(p.T, p.H), dz @ p.w64, err @ p.w64.abs() + product_bound(dz.abs() + err, p.w64), "dX")]
    if p.trans:
        got = dW[:p.V * p.H].view(p.V, p.H)
    else:
        got = torch.empty(p.H, p.V, dtype=torch.bfloat16, device="cuda")
        ccl.ccl_repack(p.m, dW, got, 1)
        got = got.t()
    pairs.append((got, dz.t() @ p.x64, err.t() @ p.x64.abs() + product_bound((dz.abs() + err).t(), p.x64), "dW"))
    for got, want, e, what in pairs:
        assert_within(got, want, e + U * (want.abs() + e) + TINY, what)
    assert ccl.ccl_gemm_status()[0] == ccl.OK


@pytest.mark.parametrize("lean", [0.0, 3.0, 8.0])
@pytest.mark.parametrize("T,V,H", [(1, 300, 64), (1, 5000, 512), (2, 1152, 520), (3, 777, 200), (4, 4096, 128), (9, 1001, 72), (15, 2503, 264), (16, 3001, 64)])
def test_row_major(T, V, H, lean):
    check(Problem(T, V, H, ignored=0.0 if T < 4 else 0.2, seed=T + V, lean=lean))


@pytest.mark.parametrize("T,V,H", [(17, 500, 64), (32, 1000, 64), (33, 1001, 1544)])
def test_one_value_each_from_17_tokens_on(T, V, H):
    Problem(T, V, H, seed=T).check_grad()


@pytest.mark.parametrize("T,V,H,P,align", [(1, 4096, 256, 4, 0), (7, 3 * 200, 72, 3, 0), (16, 2 * 1000, 136, 2, 4096), (5, 512, 128, 1, 0), (13, 1048, 40, 1, 0), (2, 4 * 648, 520, 4, 256)])
def test_strips(T, V, H, P, align):
    check(Problem(T, V, H, P, trans=False, align=align, seed=T, ignored=0.0 if T < 4 else 0.2))


@pytest.mark.parametrize("ctas,bn", [(1, 128), (1, 256), (2, 128), (2, 256)])
def test_every_tile(ctas, bn):
    with forced(ctas=ctas, bn=bn):
        check(Problem(9, 20011, 64, seed=5))
        check(Problem(16, 3001, 1600, seed=6))


def test_wanted_outputs_only_and_the_same_bits():
    p = Problem(6, 900, 64, seed=2)
    dX, dW = p.grad()
    again = p.grad()
    assert torch.equal(dX, p.grad(dw=False)[0]) and torch.equal(dW, p.grad(dx=False)[1])
    assert torch.equal(dX, again[0]) and torch.equal(dW, again[1])
    p = Problem(6, 900, 64, seed=2, ignored=1.0)
    dX, dW = p.grad()
    assert (dX[:-64] == 0).all() and (dW[:-64] == 0).all()


def test_replayed_with_other_inputs_beside_a_call():
    T, V, H = 11, 2003, 136
    a, b = Problem(T, V, H, seed=3), Problem(T, V, H, seed=4)
    want = [t.clone() for t in b.grad()]
    x, w, tg, lse, dl = a.x.clone(), a.w.clone(), a.tg.clone(), a.lse.float(), a.dloss.clone()
    dX, dW = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(ccl.ccl_linear_xent_grad_workspace(a.d), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ccl.ccl_linear_xent_grad(a.d, x, w, tg, lse, dl, dX, dW, ws)
    for t, s in ((x, b.x), (w, b.w), (tg, b.tg), (lse, b.lse.float()), (dl, b.dloss)):
        t.copy_(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph.replay()
    again = b.grad()                                            # (on the current stream, a workspace of its own)
    torch.cuda.synchronize()
    assert torch.equal(dX.view(-1), want[0][:T * H]) and torch.equal(dW.view(-1), want[1][:V * H])
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
