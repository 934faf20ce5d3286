"""An update of no tensors is a call like any other: nothing is launched, its scalars are taken as they are in any step."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import ffn

pytestmark = pytest.mark.gpu


def test_no_tensors():
    step, scale = torch.ones(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    tensors = ccl.AdamwTensors([], [], [], [])
    before = ccl.lib().ccl_launch_count()
    ccl.ccl_adamw(ccl.AdamwDesc(), tensors)
    ccl.ccl_adamw(ccl.AdamwDesc(), tensors, grad_scale=scale, step=step, lr=scale)
    assert ccl.lib().ccl_launch_count() == before
    with pytest.raises(ValueError):
        ccl.ccl_adamw(ccl.AdamwDesc(), tensors, step=step.cpu())


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_of_no_weights(bits):
    optimizer = ffn.AdamW({}, bits=bits)
    optimizer.step({})
    assert int(optimizer.t) == 1
