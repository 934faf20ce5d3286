"""The precision of ccl_linear_xent's logits with few tokens, where nothing averages what the accumulators lose.

One class: lse is the row's only logit.  Positive products, so that a sum's magnitude is its size.  An accumulator takes 256 of K in 16 additions,
each cutting off less than a unit in the last place, 2^-23 of the sum so far at most and half of that on average: 16 additions of sums that grow from a
16th to the whole, 8.5 / 2 * 2^-23 = 4.25 * 2^-23 of the logit on average.  The H / 256 accumulators are added and the result rounded to nearest:
errors of both signs, 2^-24 each and smaller while the sum is; on average below 1.1 * 2^-23 in all, with the factor log2 e's 2^-26.
Mean over the rows: 5.5 * 2^-23.
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_gemm_epilogue import workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("T,H", [(19, 1024), (128, 1024), (33, 2048), (128, 8192), (100, 1544)])
def test_mean_error_of_few_rows(T, H, trans):
    g = torch.Generator(device="cuda").manual_seed(H + T)
    V = 1 if trans else 8
    x = (1 + torch.rand(T, H, generator=g, device="cuda")).bfloat16()
    w = (1 + torch.rand(H, generator=g, device="cuda")).mul_(8.0 / H).bfloat16()
    z = x.double() @ w.double()
    if trans:
        W = w[None].contiguous()
    else:                                                       # (eight classes, seven of them far below)
        W = torch.zeros(H, V, dtype=torch.bfloat16, device="cuda")
        W[:, 3], W[:, :3], W[:, 4:] = w, -w[:, None] * 4, -w[:, None] * 4
    targets = torch.full((T,), 0 if trans else 3, dtype=torch.int32, device="cuda")
    d = ccl.XentDesc(T, V, H, None if trans else ccl.Mat(H, V, 2), w_trans=int(trans))
    lse = torch.empty(T, device="cuda")
    ccl.ccl_linear_xent(d, x, W, targets, None, lse, workspace(ccl.ccl_linear_xent_workspace(d)))
    assert float(((lse.double() - z).abs() / z).mean()) <= 5.5 * 2.0 ** -23
