"""The sizes that the binding keeps by descriptor: right for every descriptor, and not more of them than it says."""
from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc


def test_kept_sizes_are_bounded_and_right(monkeypatch):
    monkeypatch.setattr(ccl, "_gemm_bytes_cache", {})
    for M in range(1, 2 * ccl.GEMM_BYTES_ENTRIES + 10):        # a new descriptor for every token count
        assert ccl._gemm_bytes(gemm_desc(M, 64, 16)) == (2 * M * 16, 2 * 16 * 64, 2 * M * 64)
        assert len(ccl._gemm_bytes_cache) <= ccl.GEMM_BYTES_ENTRIES
    d = gemm_desc(5, 64, 16)
    assert ccl._gemm_bytes(d) is ccl._gemm_bytes(gemm_desc(5, 64, 16))
