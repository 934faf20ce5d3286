"""ccl_moe_tokens in a row on one workspace: launches in the stream together, and in a replayed graph, for both ways the grid meets
(up to 8 tokens, and more), hand the workspace's flags, counters and choice over to each other."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_moe_tokens import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 8, 9, 20, 64])
def test_launches_in_the_stream_together(T):
    x, wr, wgu, wd, res = make(T, 32, 1024, 256, 3)
    y0, _, _ = run(x, wr, wgu, wd, res, 4, True)
    other = x.flip(1).contiguous()
    y1, _, _ = run(other, wr, wgu, wd, res, 4, True)
    d = ccl.MoeDesc(T, 32, 4, 1024, 256)
    ws = torch.full((ccl.ccl_moe_tokens_workspace(d),), 0xA5, dtype=torch.uint8, device="cuda")
    ys = [torch.empty_like(res) for _ in range(20)]
    for i, y in enumerate(ys):                                # no synchronisation in between
        ccl.ccl_moe_tokens(d, other if i % 2 else x, wr, wgu, wd, y, ws, residual=res)
    assert all(torch.equal(y, y1 if i % 2 else y0) for i, y in enumerate(ys))
    assert ccl.ccl_gemm_status()[0] == ccl.OK


@pytest.mark.parametrize("T", [1, 9, 64])
def test_replayed_graph(T):
    x, wr, wgu, wd, res = make(T, 32, 1024, 256, 4)
    y0, _, _ = run(x, wr, wgu, wd, res, 4, True)
    d = ccl.MoeDesc(T, 32, 4, 1024, 256)
    ws = torch.full((ccl.ccl_moe_tokens_workspace(d),), 0xA5, dtype=torch.uint8, device="cuda")
    ys = [torch.empty_like(res) for _ in range(3)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for y in ys:
            ccl.ccl_moe_tokens(d, x, wr, wgu, wd, y, ws, residual=res)
    for _ in range(4):
        for y in ys:
            y.zero_()
        g.replay()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, y0) for y in ys)
    assert ccl.ccl_gemm_status()[0] == ccl.OK
