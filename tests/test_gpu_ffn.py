"""The feed-forward example end to end: a block's forward and backward pass against 64-bit autograd, decode steps against the layer's formula.

Tolerance: a result passes through at most four roundings to bf16 on its way (pre-activation, activation, gradient, output), each
off by at most 2^-8 of the value rounded, which later sums average: 4 * 2^-8 in the 2-norm."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import ffn
from ffn_reference import act

pytestmark = pytest.mark.gpu


def normal(*shape, std=1.0):
    return (torch.randn(*shape, device="cuda") * std).to(torch.bfloat16)


def near(got, want):
    got, want = got.double(), want.double()
    assert float((got - want).norm() / want.norm()) <= 4 * 2.0 ** -8


@pytest.mark.parametrize("T,H,I,strips,name", [(200, 256, 512, 4, "gelu_tanh"), (96, 264, 520, 1, "silu"), (1, 128, 256, 2, "gelu_erf"), (520, 512, 1024, 2, "relu")])
def test_block(T, H, I, strips, name):
    torch.manual_seed(T)
    w1, b1, w2, b2, x, dy = normal(H, I, std=0.1), normal(I, std=0.5), normal(I, H, std=0.1), normal(H, std=0.5), normal(T, H), normal(T, H)
    block = ffn.Block(w1, b1, w2, b2, T, act=getattr(ccl, "ACT_" + name.upper()), strips=strips)
    y = block.forward(x)
    g = block.backward(x, dy)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
    v = [t.double().requires_grad_(True) for t in (x, w1, b1, w2, b2)]
    want = v[0] + act(v[0] @ v[1] + v[2], name) @ v[3] + v[4]
    near(y, want.detach())
    for got, ref in zip((g["dx"], g["dw1"], g["db1"], g["dw2"], g["db2"]), torch.autograd.grad(want, v, dy.double())):
        near(got, ref)


def test_moe_layer_in_place_over_several_batch_sizes():
    torch.manual_seed(1)
    E, H, I, k = 16, 512, 256, 3
    router, gu, down = normal(E, H, std=0.1), normal(E, 2 * I, H, std=0.05), normal(E, H, I, std=0.05)
    layer = ffn.MoeLayer(router, gu, down, k)
    for T in (1, 5, 40, 5):
        x = normal(T, H)
        p = torch.softmax(x.double() @ router.double().t(), 1)
        w, ids = p.topk(k, 1)
        w = w / w.sum(1, keepdim=True)
        a = torch.einsum("tkih,th->tki", gu.double()[ids], x.double())
        want = x.double() + torch.einsum("tkhi,tki,tk->th", down.double()[ids], act(a[..., :I], "silu") * a[..., I:], w)
        layer.step(x, out=x)
        near(x, want)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
