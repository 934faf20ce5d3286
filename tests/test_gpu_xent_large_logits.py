"""ccl_linear_xent up to the largest logits it takes, 2^30 in magnitude.

Bound: the logits are single products of bf16 values, exact.  A row's sum of exponentials stands about its largest logit times log2 e rounded to fp32; the
rounding (64 at most) is in the sum's exponents and comes back with its logarithm, so that lse is off by its own rounding, 2^-24 of itself, the loss by
that and its own, and both by 2^-20 for exponentials, additions and the logarithm of their sum.  The factor log2 e = 1.44269504088896 is
1.44269502162933 in fp32, 1.335e-8 of itself less, and the logarithm is taken back by ln 2 = 1 / log2 e: lse is that much of itself less, which
is below 2^-26 = 1.49e-8.
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_gemm_epilogue import workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("top", [2.0 ** 10, 2.0 ** 20, 2.0 ** 29])
@pytest.mark.parametrize("T,V,H", [(1, 5, 8), (40, 700, 64), (300, 3001, 1544)])
def test_large_logits(T, V, H, top, sign):
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    x[:, 5] = sign * top * (1 + 0.99 * torch.rand(T, generator=g, device="cuda"))       # from top to less than twice as much
    w[:, 5] = 1.0
    w[V // 2:, 5] = 1.0 - 2.0 ** -8                             # two groups of classes
    targets = (torch.arange(T, device="cuda", dtype=torch.int32) * 7) % V
    d = ccl.XentDesc(T, V, H)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ccl.ccl_linear_xent(d, x, w, targets, loss, lse, workspace(ccl.ccl_linear_xent_workspace(d)))
    z = x.double() @ w.double().T
    want = torch.logsumexp(z, 1)
    at = z.gather(1, targets.long()[:, None])[:, 0]
    bound = (2.0 ** -24 + 2.0 ** -26) * want.abs() + 2.0 ** -20
    assert ((lse.double() - want).abs() <= bound).all()
    assert ((loss.double() - (want - at)).abs() <= bound + 2.0 ** -24 * (want - at).abs()).all()
    assert ccl.ccl_gemm_status()[0] == ccl.OK
