"""ccl_linear_xent_grad where the gradient of the losses is at the ends of fp32's range: the gradients are linear in it.

Bounds (u = 2^-8): the formula in 64 bits with the kernel's own lse.  dz is off by u |dz| and by 2^-20 + 2 e (|z| + |lse|) of p |dloss|, which is less than
u of it, so a gradient by 2 u of the sum of magnitudes of its terms and, rounded itself, by u of its value.  Below 2^-126, the least normal number of
fp32 and of bf16, values may be flushed to zero, where they are sums of T or V of them each may be: 2^-126 for the output.
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_gemm_epilogue import workspace

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


@pytest.mark.parametrize("dloss", [1e-44, 1e-40, 2.0 ** -127, 2.0 ** -126, 1e-30, 1e30, 2.0 ** 126])
@pytest.mark.parametrize("T,V,H", [(33, 500, 64), (300, 1001, 256)])
def test_range_of_dloss(T, V, H, dloss):
    g = torch.Generator(device="cuda").manual_seed(0)
    x = (torch.randn(T, H, generator=g, device="cuda") * 0.1).bfloat16()
    w = (torch.randn(V, H, generator=g, device="cuda") * 0.1).bfloat16()
    targets = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    d = ccl.XentDesc(T, V, H)
    loss, lse = (torch.empty(T, device="cuda") for _ in range(2))
    ccl.ccl_linear_xent(d, x, w, targets, loss, lse, workspace(ccl.ccl_linear_xent_workspace(d)))
    dl = torch.full((T,), dloss, device="cuda")
    dl[::3] = 0.0                                                    # rows without a gradient beside them
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ccl.ccl_linear_xent_grad(d, x, w, targets, lse, dl, dx, dw, workspace(ccl.ccl_linear_xent_grad_workspace(d)))
    z = x.double() @ w.double().T
    dz = torch.exp(z - lse.double()[:, None])
    dz[torch.arange(T, device="cuda"), targets.long()] -= 1.0
    dz *= dl.double()[:, None]
    for got, a, b in ((dx, dz, w.double()), (dw, dz.T, x.double())):
        want, sizes = a @ b, a.abs() @ b.abs()
        assert torch.isfinite(got).all()
        assert ((got.double() - want).abs() <= 2 * U * sizes + U * want.abs() + 2.0 ** -126).all()
