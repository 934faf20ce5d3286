"""gelu (tanh) and silu where their value is small beside their argument: what is stored keeps bf16's relative precision there, the slopes'
as well.

Both are z s(t) with the logistic function s(t) = 1 / (1 + 2^(-t log2 e)): t = z, or t = 2 sqrt(2/pi) (z + 0.044715 z^3).  The exponent's
argument is built with at most six fp32 roundings (of constants, of z^2, of the sum and of products), each off by at most 2^-24 of it: 2^-21 |t|
of the value covers them; exponential, reciprocal and products: 2^-19 of it.  The slopes s + z s (1 - s) dt/dz are sums of two such terms.
Then one rounding to bf16, u = 2^-8.  z goes down to where the exponential is still a normal fp32 number."""
import math

import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc
from ffn_reference import U, assert_within

pytestmark = pytest.mark.gpu

A, B = 2 * math.sqrt(2 / math.pi), 0.044715


def arguments(lowest):
    """The bf16 values from `lowest` to -2^-6."""
    z = torch.arange(0x3C80, 0x7F80, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    z = -z[z <= -lowest]
    return z[z.numel() % 8:].clone()                          # (a base of its own, aligned)


def parts(z, name):
    """t, dt/dz, s and 1 - s in 64 bits."""
    x = z.double()
    t, dt = (x, torch.ones_like(x)) if name == "silu" else (A * (x + B * x ** 3), A * (1 + 3 * B * x * x))
    return x, t, dt, 1 / (1 + torch.exp(-t)), 1 / (1 + torch.exp(t))


@pytest.mark.parametrize("name,lowest", [("gelu_tanh", -9.5), ("silu", -80.0)])
def test_value(name, lowest):
    z = arguments(lowest)
    M, N, K = 40, z.numel(), 8
    d = gemm_desc(M, N, K)
    c = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    a, b = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(K, N, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(16, ccl.ccl_gemm_epilogue_workspace(d)), dtype=torch.uint8, device="cuda")
    ccl.ccl_gemm_epilogue(d, a, b, c, ws, act=getattr(ccl, "ACT_" + name.upper()), bias=z)
    x, t, _, s, _ = parts(z, name)
    want = x * s
    assert_within(c, want.expand(M, N), want.abs() * (U + 2.0 ** -19 + 2.0 ** -21 * t.abs()) * (1 + U), name)
    assert ccl.ccl_gemm_status()[0] == ccl.OK


@pytest.mark.parametrize("name,lowest", [("gelu_tanh", -9.5), ("silu", -80.0)])
def test_slope(name, lowest):
    z = arguments(lowest)
    M, N = 3, z.numel()
    dy = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    dz = torch.empty_like(dy)
    ccl.ccl_bias_act_grad(ccl.Mat(M, N, 2), dy, z.expand(M, N).contiguous(), dz, act=getattr(ccl, "ACT_" + name.upper()))
    x, t, dt, s, rest = parts(z, name)
    want = s + x * s * rest * dt
    err = (s + (x * s * rest * dt).abs()) * 2 * (2.0 ** -19 + 2.0 ** -21 * t.abs())
    assert_within(dz, want.expand(M, N), err + U * (want.abs() + err), name)
