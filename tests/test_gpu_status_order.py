"""ccl_gemm_status with several reports at once: an expired wait is told before bad offsets or a bad target, which only mean that a row was left out."""
import numpy as np
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc
from test_gpu_gemm_epilogue import workspace

pytestmark = pytest.mark.gpu


def bad_target():
    T, V, H = 8, 100, 64
    d = ccl.XentDesc(T, V, H)
    x, w = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    targets = torch.zeros(T, dtype=torch.int32, device="cuda")
    targets[3] = V
    loss = torch.empty(T, device="cuda")
    ccl.ccl_linear_xent(d, x, w, targets, loss, None, workspace(ccl.ccl_linear_xent_workspace(d)))


def bad_offsets():
    N, K = 512, 256
    d = gemm_desc(64, N, K, 1, ("row", "row", "row"), 0, 0, 0, 1)
    a, b, c = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in (64 * K, N * K, 64 * N))
    ccl.ccl_gemm_grouped(d, 1, 16, torch.from_numpy(np.array([0, 40], dtype=np.int32)).cuda(), a, b, 0, c)      # 40 rows, 16 allowed


@pytest.mark.parametrize("which,code", [(0, 6), (1, 101)])
@pytest.mark.parametrize("bad,detail", [(bad_target, 10), (bad_offsets, 5)])
def test_expired_wait_comes_first(which, code, bad, detail):
    ccl.ccl_gemm_status()
    src = torch.arange(2048, dtype=torch.uint8, device="cuda")
    for first, second in ((lambda: ccl.ccl_selftest_wait_timeout(which, 1000, src), bad), (bad, lambda: ccl.ccl_selftest_wait_timeout(which, 1000, src))):
        first()
        second()
        assert ccl.ccl_gemm_status() == (ccl.ERR_TIMEOUT, code)
        assert ccl.ccl_gemm_status() == (ccl.OK, 0)
    bad()
    assert ccl.ccl_gemm_status() == (ccl.ERR_SHAPE, detail)
    assert ccl.ccl_gemm_status() == (ccl.OK, 0)
