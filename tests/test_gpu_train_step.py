"""A training step put together -- normalisation, feed-forward block, loss over a vocabulary, their gradients and the update -- against 64-bit
autograd of the whole, and captured into a graph.

Tolerance: a gradient passes through at most eight roundings to bf16 on its way (normalised x, pre-activation, activation, block's output, dz of
the loss, dy, gradient of the activation, gradient of the normalised x) and its own, each off by at most 2^-8 of the value rounded, which
later sums average: 9 * 2^-8 in the 2-norm."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import ffn
from ffn_reference import act
from test_gpu_adamw import plain, same

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def normal(*shape, std=1.0):
    return (torch.randn(*shape, device="cuda") * std).to(torch.bfloat16)


def near(got, want, what):
    got, want = got.double(), want.double()
    off = float((got - want).norm() / want.norm())
    assert off <= 9 * 2.0 ** -8, f"{what}: {off:.2e}"


def setup(T, H, I, V, strips, name, layer, bits=32):
    torch.manual_seed(T + V)
    w = {"w1": normal(H, I, std=0.1), "b1": normal(I, std=0.3), "w2": normal(I, H, std=0.1), "b2": normal(H, std=0.3), "gamma": 1 + normal(H, std=0.2),
         "beta": normal(H, std=0.2) if layer else None, "vocabulary": normal(V, H, std=0.1)}
    kind = ccl.NORM_LAYER if layer else ccl.NORM_RMS
    block = ffn.Block(w["w1"], w["b1"].clone(), w["w2"].clone(), w["b2"].clone(), T, act=getattr(ccl, "ACT_" + name.upper()), strips=strips,
                      norm=(w["gamma"].clone(), w["beta"].clone() if layer else None), kind=kind)
    head = ffn.Head(w["vocabulary"].clone(), T)
    x = normal(T, H)
    targets = torch.randint(0, V, (T,), device="cuda")
    live = torch.rand(T, device="cuda") > 0.2
    live[0] = True
    tg = torch.where(live, targets, -100).to(torch.int32)
    dloss = (torch.rand(T, device="cuda") + 0.5) / T
    optimizer = ffn.AdamW({**block.weights(), "vocabulary": head.w}, bits=bits, **HYPER)
    return w, block, head, optimizer, x, targets, live, tg, dloss


def reference(w, x, targets, live, dloss, name, layer):
    v = {k: t.double().requires_grad_(True) for k, t in {**w, "x": x}.items() if t is not None}
    c = v["x"] - v["x"].mean(1, keepdim=True) if layer else v["x"]
    n = c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5) * v["gamma"]
    if layer:
        n = n + v["beta"]
    y = v["x"] + act(n @ v["w1"] + v["b1"], name) @ v["w2"] + v["b2"]
    z = y @ v["vocabulary"].t()
    loss = (torch.logsumexp(z, 1) - z.gather(1, targets[:, None])[:, 0]) * live
    grads = torch.autograd.grad((loss * dloss.double()).sum(), list(v.values()))
    return loss.detach(), dict(zip(v, grads))


@pytest.mark.parametrize("T,H,I,V,strips,name,layer", [(200, 256, 512, 1001, 4, "gelu_tanh", True), (96, 264, 520, 333, 1, "silu", False), (1, 128, 256, 50, 2, "gelu_erf", True),
                                                       (520, 512, 1024, 5000, 2, "silu", True)])
def test_gradients_of_the_whole(T, H, I, V, strips, name, layer):
    w, block, head, _, x, targets, live, tg, dloss = setup(T, H, I, V, strips, name, layer)
    y = block.forward(x)
    loss = head.loss(y, tg)
    dy, dw = head.backward(y, tg, dloss)
    got = block.backward(x, dy)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
    want_loss, want = reference(w, x, targets, live, dloss, name, layer)
    near(loss, want_loss, "loss")
    near(dw, want["vocabulary"], "dw")
    for k in ("x", "w1", "b1", "w2", "b2", "gamma") + (("beta",) if layer else ()):
        near(got["d" + k], want[k], "d" + k)
    if not layer:
        assert got["dbeta"] is None


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_update_every_weight(bits):
    T, H, I, V = 130, 128, 256, 700
    w, block, head, optimizer, x, _, _, tg, dloss = setup(T, H, I, V, 2, "silu", True, bits)
    masters = dict(zip(optimizer.names, optimizer.masters))
    for t in (1, 2):
        before = {k: m.clone() for k, m in masters.items()}
        states = {k: (optimizer.m[i].clone(), optimizer.v[i].clone()) + (() if bits == 32 else (optimizer.scales[0][i].clone(), optimizer.scales[1][i].clone()))
                  for i, k in enumerate(optimizer.names)}
        y = block.forward(x)
        head.loss(y, tg)
        dy, dw = head.backward(y, tg, dloss)
        grads = block.backward(x, dy, stored=True)
        grads = {**{k: grads["d" + k] for k in block.weights()}, "vocabulary": dw}
        ffn.train_step(block, head, optimizer, x, tg, dloss)
        for i, k in enumerate(optimizer.names):
            s = states[k]
            m, v = (s[0].view(-1), s[1].view(-1)) if bits == 32 else ((s[0].view(-1), s[2]), (s[1].view(-1), s[3]))
            p, _, _ = plain(before[k].view(-1), grads[k].view(-1), m, v, t, **HYPER)
            # (the factors of the step's number come from the device's 64-bit power here and from the host's there: a last place)
            assert (masters[k].view(-1) - p).abs().max() <= 2.0 ** -22 * p.abs().max(), k
            same(optimizer.weights[i], masters[k].to(torch.bfloat16), k)
            assert not torch.equal(before[k], masters[k]), k
    assert block.w1.data_ptr() == optimizer.weights[0].data_ptr() and int(optimizer.t) == 2


def test_captured_step():
    T, H, I, V = 64, 128, 256, 500
    a = setup(T, H, I, V, 2, "gelu_tanh", True)
    b = setup(T, H, I, V, 2, "gelu_tanh", True)
    _, block, head, optimizer, x, _, _, tg, dloss = a
    ffn.train_step(block, head, optimizer, x, tg, dloss)          # (what a first call sets up)
    xs = [normal(T, H) for _ in range(4)]
    buf = x.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = ffn.train_step(block, head, optimizer, buf, tg, dloss)
    _, block2, head2, optimizer2, _, _, _, tg2, dloss2 = b
    ffn.train_step(block2, head2, optimizer2, x, tg2, dloss2)
    for xi in xs:
        buf.copy_(xi)
        g.replay()
        want = ffn.train_step(block2, head2, optimizer2, xi, tg2, dloss2)
        torch.cuda.synchronize()
        assert torch.equal(loss, want)
    for p, q in zip(optimizer.masters, optimizer2.masters):
        same(p, q, "weights after five steps")
    assert ccl.ccl_gemm_status()[0] == ccl.OK
