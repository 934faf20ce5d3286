"""The expiry path of ccl_moe_tokens' meetings: a meeting that waits, with a limit of a millisecond, for one CTA more than there are.  The
kernel ends by itself and reports it once, and the workspace is left with no flag that the launch, replayed with the same
mark, would take for a CTA's arrival."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_moe_tokens import make, run


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 4, 20])
@pytest.mark.parametrize("meeting", [1, 2])
def test_a_meeting_that_does_not_come_about(T, meeting):
    E_, topk, H, I = 16, 2, 256, 64
    x, wr, wgu, wd, res = make(T, E_, H, I, 6)
    y0, _, _ = run(x, wr, wgu, wd, None, topk, True)
    d = ccl.MoeDesc(T, E_, topk, H, I)
    ws = torch.full((ccl.ccl_moe_tokens_workspace(d),), 0xA5, dtype=torch.uint8, device="cuda")
    y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    ccl.ccl_selftest_moe_timeout(d, x, wr, wgu, wd, y, ws, meeting, 1000)
    st, detail = ccl.ccl_gemm_status()
    assert st == ccl.ERR_TIMEOUT and detail in (8, 9), (st, detail)
    assert ccl.ccl_gemm_status() == (ccl.OK, 0)               # reported once
    # the workspace: logits, a flag per CTA, sixteen words of nothing, the word that ends the first meeting
    ctas = torch.cuda.get_device_properties(0).multi_processor_count & ~1
    words = ws[(T * E_ * 4 + 127) // 128 * 128:][: (ctas + 17) * 8].view(torch.int64)
    assert (words[:ctas] == 0).all() and words[ctas + 16] == 0
    ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws)              # the same workspace serves the next call
    assert ccl.ccl_gemm_status()[0] == ccl.OK
    assert torch.equal(y, y0)


def test_refusals():
    d = ccl.MoeDesc(4, 16, 2, 64, 32)
    p = [i << 12 for i in range(1, 7)]
    for meeting, limit in ((0, 1000), (3, 1000), (1, 0), (2, 10 ** 6)):
        assert ccl.lib().ccl_selftest_moe_timeout(d, *p, 1 << 20, meeting, limit, None) == ccl.ERR_INVALID_ARG
    assert ccl.lib().ccl_selftest_moe_timeout(d, *p, 16, 1, 1000, None) == ccl.ERR_WORKSPACE
