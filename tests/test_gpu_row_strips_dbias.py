"""The bias's gradient of ccl_gemm_act_grad where the rows are in strips of which the last has fewer tile rows than the others: the tile
grid has places without rows there, and the workspace (full of NaN before the call) must not reach the sums through them.
Tolerances: ffn_reference.py."""
import pytest

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc
from test_gpu_gemm_epilogue import check_forward, check_grad, forced

# M, N, K, P: strips of ceil(M / P) rows.  With tiles of 128 rows (one CTA) or 256 (a pair) the last strip has a tile row less than the
# others where its height crosses a multiple of that.
CASES = [
    (257, 512, 512, 2, 1),       # 129 + 128
    (646, 512, 128, 5, 1),       # 130 x 4 + 126
    (388, 512, 128, 3, 1),       # 130 + 130 + 128
    (1286, 512, 136, 5, 2),      # 258 x 4 + 254
    (1025, 1032, 328, 2, 2),     # 513 + 512
    (3077, 264, 128, 6, 2),      # 513 x 5 + 512
]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,P,ctas", CASES)
@pytest.mark.parametrize("lay", [("ccl", "row", "ccl"), ("row", "row", "ccl"), ("ccl", "row", "row")], ids=["A-and-C", "C", "A"])
def test_a_last_strip_with_fewer_tile_rows(M, N, K, P, ctas, lay):
    for v in (dict(), dict(ctas=ctas, bn=128), dict(ctas=ctas, bn=256)):
        with forced(**v):
            d = gemm_desc(M, N, K, P, lay, 0, 0, 1, 1)
            check_grad(M, N, K, "gelu_tanh", d, 0, 0, seed=11)
            check_grad(M, N, K, "none", d, 0, 0, seed=12)
            check_forward(M, N, K, "silu", d, 0, 0, seed=13)


def test_the_workspace_counts_tile_rows_that_exist():
    """A line of 512 fp32 sums for every 32 rows of every tile row (no GPU: the plan of tiles of 128 rows)."""
    with forced(ctas=1, bn=128):
        for M, P, tile_rows in ((258, 2, 4), (257, 2, 3), (646, 5, 9), (388, 3, 5)):
            d = gemm_desc(M, 512, 128, P, ("ccl", "row", "ccl"), 0, 0, 1, 1)
            assert ccl.ccl_gemm_act_grad_workspace(d) == tile_rows * 4 * 512 * 4
