"""One MoeLayer stepped on several streams: no two steps that can overlap share a workspace."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import ffn

pytestmark = pytest.mark.gpu


def layer(E=16, H=512, I=256, k=3):
    torch.manual_seed(2)
    normal = lambda *shape, std: (torch.randn(*shape, device="cuda") * std).to(torch.bfloat16)   # noqa: E731
    return ffn.MoeLayer(normal(E, H, std=0.1), normal(E, 2 * I, H, std=0.05), normal(E, H, I, std=0.05), k), normal(8, 5, H, std=1.0)


def test_a_step_has_a_workspace_of_its_own(monkeypatch):
    moe, xs = layer()
    held = []
    monkeypatch.setattr(ccl, "ccl_moe_tokens", lambda d, x, wr, gu, dn, y, ws, residual=None: held.append(ws))
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        with torch.cuda.stream(s):
            moe.step(xs[0])
    assert len({w.data_ptr() for w in held}) == len(streams)   # (all three are still referenced)
    assert all(w.nbytes >= ccl.ccl_moe_tokens_workspace(ccl.MoeDesc(5, 16, 3, 512, 256)) for w in held)


def test_streams_interleaved():
    moe, xs = layer()
    want = [moe.step(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for turn in range(24):
        with torch.cuda.stream(streams[turn % 3]):
            got.append((turn % 8, moe.step(xs[turn % 8])))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i, y in got)
    assert ccl.ccl_gemm_status()[0] == ccl.OK


def test_captured_step():
    moe, xs = layer()
    want = moe.step(xs[1])
    x, y = xs[0].clone(), torch.empty_like(xs[0])
    moe.step(x, out=y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moe.step(x, out=y)
    x.copy_(xs[1])
    for _ in range(3):
        moe.step(xs[2])                                        # calls outside the graph in between
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
