"""8-bit states whose values leave fp32: a block with an infinite moment or root is NaN from then on, as one with a NaN is, and no other block is."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from test_gpu_adamw import HYPER, State, decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [1e20, -3e38, float("inf"), float("-inf")])
@pytest.mark.parametrize("n", [1000, 700])
def test_block_with_an_infinite_state_is_nan(n, value):
    s = State([n], 8, True, seed=2)
    s.g[0].fill_(1e-3)
    s.g[0][300] = value                                         # (1e20 and 3e38 are finite: only their squares are not)
    ccl.ccl_adamw(ccl.AdamwDesc(step=1, **HYPER), s.tensors())
    block = list(range(256, 512))
    assert torch.isnan(decode(s.v[0], s.vs[0])).nonzero().flatten().tolist() == block
    assert torch.isnan(decode(s.m[0], s.ms[0])).nonzero().flatten().tolist() == ([] if abs(value) < float("inf") else block)
    s.g[0].fill_(1e-3)
    for t in (2, 3):
        ccl.ccl_adamw(ccl.AdamwDesc(step=t, **HYPER), s.tensors())
        assert torch.isnan(s.p[0]).nonzero().flatten().tolist() == block
        assert torch.isnan(decode(s.v[0], s.vs[0])).nonzero().flatten().tolist() == block
