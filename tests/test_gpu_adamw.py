"""ccl_adamw against the same operations one by one (the same bits), and against the update's definition in 64 bits.

Bounds of the comparison in 64 bits, per step and relative to the magnitudes summed (e = 2^-24, half an ulp of fp32): m and v are three roundings
and two rounded factors of a sum: 5 e of |b1 m| + |(1 - b1) g| (v: 6 e); p: the two factors, product, quotient (root, product, sum, division) and
difference: 4 e |p| + 16 e |lr step|."""
import math

import pytest
import torch

from paper_2606_11718_b200 import binding as ccl

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def scales_of(x):
    """x in rows of 256 -> (scale, reciprocal) of each row, in the stated operations"""
    top = x.abs().amax(1)
    kept = ~(top < 1e-30)
    zero = torch.zeros_like(top)
    return torch.where(kept, top * (1 / 448), zero), torch.where(kept, torch.div(torch.full_like(top, 448.0), top), zero)


def rows256(t):
    return torch.nn.functional.pad(t, (0, -t.numel() % 256)).view(-1, 256)


def encode(t, root):
    x = rows256(t)
    scale, inv = scales_of(x)
    q = (x * inv[:, None]).to(F8)
    if root:
        q = torch.where((x > 0) & (q.float() == 0), torch.tensor(2.0 ** -9, device=t.device), q.float()).to(F8)
    return q.view(-1)[:t.numel()].clone(), scale


def decode(q, scale):
    return (rows256(q.float()) * scale[:, None]).reshape(-1)[:q.numel()]


def plain(p, g, m, v, t, gscale=None, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1):
    """One tensor's step, every operation a rounding of its own; m, v: float32, or (e4m3, scales).  Returns p, m, v, in the given forms."""
    g = g.float() if gscale is None else g.float() * gscale
    eight = isinstance(m, tuple)
    m0 = decode(*m) if eight else m
    v0 = decode(*v) if eight else v
    if eight:
        v0 = v0 * v0
    m1 = m0 * beta1 + g * (1 - beta1)
    v1 = v0 * beta2 + g * (1 - beta2) * g
    r = torch.sqrt(v1)
    step = torch.div(m1, r * (1 / math.sqrt(1 - beta2 ** t)) + eps)
    p = p * (1 - lr * weight_decay) - step * (lr / (1 - beta1 ** t))
    return (p, encode(m1, False), encode(r, True)) if eight else (p, m1, v1)


def same(a, b, what):
    a, b = a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)
    assert torch.equal(a, b), f"{what}: {int((a != b).sum())} bytes differ"


class State:
    def __init__(self, sizes, bits, wide, copy=True, seed=0, shift=0, std=1e-3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda n, s: torch.randn(n + shift, generator=g, device="cuda")[shift:] * s if not shift else \
            torch.cat([torch.zeros(shift, device="cuda"), torch.randn(n, generator=g, device="cuda") * s])[shift:]      # noqa: E731
        cast = lambda t, dt: torch.cat([torch.zeros(shift, device="cuda", dtype=dt), t.to(dt)])[shift:]                   # noqa: E731
        self.bits = bits
        self.p = [normal(n, 0.02) for n in sizes]
        self.g = [normal(n, std) if wide else cast(normal(n, std), torch.bfloat16) for n in sizes]
        self.copy = [cast(torch.zeros(n, device="cuda"), torch.bfloat16) for n in sizes] if copy else None
        if bits == 32:
            self.m = [torch.zeros(n + shift, device="cuda")[shift:] for n in sizes]
            self.v = [torch.zeros(n + shift, device="cuda")[shift:] for n in sizes]
            self.ms = self.vs = None
        else:
            self.m = [torch.zeros(n + shift, device="cuda", dtype=F8)[shift:] for n in sizes]
            self.v = [torch.zeros(n + shift, device="cuda", dtype=F8)[shift:] for n in sizes]
            self.ms = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]
            self.vs = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]

    def tensors(self):
        return ccl.AdamwTensors(self.p, self.g, self.m, self.v, copies=self.copy, m_scales=self.ms, v_scales=self.vs)

    def parts(self, i):
        if self.bits == 32:
            return self.p[i].clone(), self.g[i], self.m[i].clone(), self.v[i].clone()
        return self.p[i].clone(), self.g[i], (self.m[i].clone(), self.ms[i].clone()), (self.v[i].clone(), self.vs[i].clone())

    def check(self, i, want):
        p, m, v = want
        same(self.p[i], p, f"p of tensor {i}")
        if self.bits == 32:
            same(self.m[i], m, f"m of tensor {i}")
            same(self.v[i], v, f"v of tensor {i}")
        else:
            for a, b, what in ((self.m[i], m[0], "m"), (self.ms[i], m[1], "m's scales"), (self.v[i], v[0], "v"), (self.vs[i], v[1], "v's scales")):
                same(a, b, f"{what} of tensor {i}")
        if self.copy is not None:
            same(self.copy[i], p.to(torch.bfloat16), f"copy of tensor {i}")


LISTS = [[1], [3, 0, 5], [255, 256, 257, 1, 4096, 4097], [100000], [7 * k + 1 for k in range(60)], [13] * 450, [3000000, 5]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s)}")
def test_three_steps_bit_for_bit(sizes, bits):
    for wide, copy, shift, clip in ((False, True, 0, None), (True, False, 0, 0.37), (False, True, 1, 0.5), (True, True, 3, None)):
        s = State(sizes, bits, wide, copy, seed=len(sizes) + bits, shift=shift)
        tensors = s.tensors()
        scale = None if clip is None else torch.tensor([clip], device="cuda")
        for t in (1, 2, 3):
            want = [plain(*s.parts(i), t, gscale=scale) for i in range(len(sizes))]
            ccl.ccl_adamw(ccl.AdamwDesc(step=t, **HYPER), tensors, grad_scale=scale)
            for i in range(len(sizes)):
                s.check(i, want[i])
            for g in s.g:
                g.mul_(-0.7)


def test_against_the_definition():
    n, h, e = 40000, HYPER, 2.0 ** -24
    s = State([n], 32, True, seed=5)
    p, m, v = s.p[0].double(), torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for t in range(1, 6):
        g = s.g[0].double()
        p, m0, v0 = s.p[0].double(), s.m[0].double(), s.v[0].double()                       # a step at a time, from the kernel's own state
        ccl.ccl_adamw(ccl.AdamwDesc(step=t, **h), s.tensors())
        m, v = h["beta1"] * m0 + (1 - h["beta1"]) * g, h["beta2"] * v0 + (1 - h["beta2"]) * g * g
        step = h["lr"] * (m / (1 - h["beta1"] ** t)) / ((v / (1 - h["beta2"] ** t)).sqrt() + h["eps"])
        want = p - h["lr"] * h["weight_decay"] * p - step
        assert ((s.m[0].double() - m).abs() <= 5 * e * ((h["beta1"] * m0).abs() + ((1 - h["beta1"]) * g).abs()) + 1e-44).all()
        assert ((s.v[0].double() - v).abs() <= 6 * e * v + 1e-44).all()
        m_rel = 5 * e * ((h["beta1"] * m0).abs() + ((1 - h["beta1"]) * g).abs()) / m.abs().clamp(min=1e-300)
        assert ((s.p[0].double() - want).abs() <= 4 * e * p.abs() + (16 * e + m_rel) * step.abs()).all()
        s.g[0].mul_(-0.9).add_(1e-4)


def test_eight_bits_stay_near_thirty_two():
    # A state decoded is off by half a step of e4m3 (2^-4 of it) or half the least value (2^-10 of the block's scale); roots are rounded up to
    # the least value at most.  After one step from zero states p does not depend on what is kept: equal bits.
    a, b = State([70000], 32, False, seed=9), State([70000], 8, False, seed=9)
    for s in (a, b):
        ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), s.tensors())
    same(a.p[0], b.p[0], "p after one step")
    top = rows256(a.m[0]).abs().amax(1)
    m = decode(b.m[0], b.ms[0])
    assert ((m - a.m[0]).abs() <= a.m[0].abs() * (2.0 ** -4 + 2.0 ** -20) + (top / 448 * 2.0 ** -10).repeat_interleave(256)[:70000] * 1.001).all()
    r, root = decode(b.v[0], b.vs[0]), a.v[0].sqrt()
    top = rows256(root).amax(1)
    assert ((r - root).abs() <= root * (2.0 ** -4 + 2.0 ** -20) + (top / 448 * 2.0 ** -9).repeat_interleave(256)[:70000] * 1.001).all()
    assert (r[root > 0] > 0).all()


def test_small_roots_never_become_zero():
    s = State([512], 8, True, seed=1)
    s.g[0].fill_(1e-9)
    s.g[0][0] = 1.0                                             # one large gradient in the first block
    s.g[0][5] = 0.0
    ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), s.tensors())
    r = decode(s.v[0], s.vs[0])
    assert (r[torch.arange(512, device="cuda") != 5] > 0).all() and r[5] == 0
    before = s.p[0].clone()
    s.g[0].zero_()
    ccl.ccl_adamw(ccl.AdamwDesc(step=2, **HYPER), s.tensors())
    assert ((s.p[0] - before).abs() < 10 * HYPER["lr"]).all()   # (a zero root under a moment of 1e-10 would be a step of 1e-2 / lr)


def test_nothing_and_non_finite():
    for bits in (32, 8):
        s = State([1000], bits, True, seed=2)
        s.g[0].zero_()
        p = s.p[0].clone()
        ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), s.tensors())
        same(s.p[0], p * (1 - HYPER["lr"] * HYPER["weight_decay"]), "decay alone")
        assert (s.m[0].view(torch.uint8) == 0).all() and (s.v[0].view(torch.uint8) == 0).all()
        s.g[0].fill_(1e-3)
        s.g[0][300] = float("nan")
        ccl.ccl_adamw(ccl.AdamwDesc(step=2, **HYPER), s.tensors())
        assert torch.isnan(s.p[0]).nonzero().flatten().tolist() == [300]
        if bits == 8:
            assert torch.isnan(decode(s.m[0], s.ms[0])).nonzero().flatten().tolist() == list(range(256, 512))
            assert torch.isnan(decode(s.v[0], s.vs[0])).nonzero().flatten().tolist() == list(range(256, 512))


def test_captured_with_step_and_rate_on_the_device():
    sizes = [5000, 77]
    for bits in (32, 8):
        a, b = State(sizes, bits, False, seed=3), State(sizes, bits, False, seed=3)
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([0.0], device="cuda")
        at, bt = a.tensors(), b.tensors()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step.add_(1)
            ccl.ccl_adamw(ccl.AdamwDesc(**HYPER), at, step=step, lr=lr)
        for t in range(1, 6):
            rate = torch.tensor([1e-3 / t])
            lr.copy_(rate)
            g.replay()
            ccl.ccl_adamw(ccl.AdamwDesc(**{**HYPER, "lr": rate.item(), "step": t}), bt)
            torch.cuda.synchronize()
            for i in range(2):
                # the factors are rounded to fp32 from 64-bit powers of two different libraries: equal but in a rare last place
                assert (a.p[i] - b.p[i]).abs().max() <= 2.0 ** -22 * b.p[i].abs().max()


def test_on_another_stream():
    s, t = State([200000], 32, False, seed=4), State([200000], 32, False, seed=4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), s.tensors())
    torch.cuda.current_stream().wait_stream(stream)
    ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), t.tensors())
    same(s.p[0], t.p[0], "p")
