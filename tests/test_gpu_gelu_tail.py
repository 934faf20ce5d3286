"""gelu (erf) where its value is small beside its argument: what is stored keeps bf16's relative precision there.

Bound: a product of a fitted polynomial (1.5e-7 of the value), its evaluation in fp32, a hardware reciprocal and a hardware exponential
(each a few units of 2^-23): 2^-19 of the value in all; the exponential's argument z^2 / 2 log2 e is the product of three rounded factors,
each off by at most 2^-24 of it: 2^-22 z^2 / 2 of the value.  Then one rounding to bf16, u = 2^-8.  z goes down to where the value's
exponential is still a normal fp32 number."""
import math

import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc
from ffn_reference import U, assert_within

pytestmark = pytest.mark.gpu


def arguments():
    """Every bf16 value in [-12.5, -2^-6], and their opposites."""
    z = torch.arange(0x3C80, 0x4149, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    assert float(z[0]) == 2.0 ** -6 and float(z[-1]) == 12.5
    z = torch.cat([-z, z])
    return z[: z.numel() // 16 * 16].contiguous()


def relative(z):
    return 2.0 ** -19 + 2.0 ** -22 * z * z / 2


def test_value():
    z = arguments()
    M, N, K = 40, z.numel(), 8
    d = gemm_desc(M, N, K)
    c = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    A, B = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(K, N, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(16, ccl.ccl_gemm_epilogue_workspace(d)), dtype=torch.uint8, device="cuda")
    ccl.ccl_gemm_epilogue(d, A, B, c, ws, act=ccl.ACT_GELU_ERF, bias=z)
    x = z.double()
    want = 0.5 * x * torch.special.erfc(-x / math.sqrt(2))
    assert_within(c, want.expand(M, N), want.abs() * (U + relative(x)), "gelu")
    assert ccl.ccl_gemm_status()[0] == ccl.OK


def test_slope():
    z = arguments()
    M, N = 3, z.numel()
    dy = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    dz = torch.empty_like(dy)
    ccl.ccl_bias_act_grad(ccl.Mat(M, N, 2), dy, z.expand(M, N).contiguous(), dz, act=ccl.ACT_GELU_ERF)
    x = z.double()
    cdf, rest = 0.5 * torch.special.erfc(-x / math.sqrt(2)), x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    want = cdf + rest
    err = (cdf + rest.abs()) * relative(x)
    assert_within(dz, want.expand(M, N), err + U * (want.abs() + err), "slope")
