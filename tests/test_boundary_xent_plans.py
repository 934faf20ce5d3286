"""The gradient's workspace follows the planner's switches, whatever was asked before.  No GPU."""
import pytest

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import build as ccl_build
from test_gpu_gemm_epilogue import forced


@pytest.fixture(scope="module", autouse=True)
def built():
    ccl_build.build()


@pytest.mark.parametrize("T,V,H", [(8192, 256, 512), (4096, 512, 1024)])
def test_workspace_follows_the_balanced_switch(T, V, H):
    d = ccl.XentDesc(T, V, H)
    plain = ccl.ccl_linear_xent_grad_workspace(d)
    with forced(balanced=1):
        cut = ccl.ccl_linear_xent_grad_workspace(d)
    assert ccl.ccl_linear_xent_grad_workspace(d) == plain
    assert cut > plain                                          # (the balanced products keep partial sums)
    with forced(balanced=1):
        assert ccl.ccl_linear_xent_grad_workspace(d) == cut
