"""Operands that the feed-forward operators' calls from Python refuse before anything is launched: workspaces and matrices that the GPU
cannot reach as they are, and matrices of another floating type, whose bytes would be read as bfloat16."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc

BF16 = torch.bfloat16


class Elsewhere:
    """What the checks look at of a tensor on another device than the current one."""
    dtype, nbytes = BF16, 1 << 20

    def is_contiguous(self):
        return True

    def get_device(self):
        return 1


def test_another_device(monkeypatch):
    for current in (0, 1):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
        if current == 1:
            assert ccl._check_operands("op", (None, 16), (Elsewhere(), 16), (Elsewhere(), 16)) == 1
            continue
        with pytest.raises(ValueError, match="current CUDA device"):
            ccl._check_operands("op", (Elsewhere(), 16))
    with pytest.raises(ValueError, match="beside the operands"):
        ccl._check_vector(Elsewhere(), 8, "bias", 0)
    with pytest.raises(ValueError, match="beside the operands"):
        ccl._check_workspace(Elsewhere(), "op", 0)
    with pytest.raises(ValueError, match="current CUDA device"):
        ccl._check_operands("op", (torch.zeros(8, dtype=BF16), 16))
    with pytest.raises(ValueError, match="current CUDA device"):
        ccl._check_operands("op", (Elsewhere(), 16), (torch.zeros(8, dtype=BF16), 16))


def gemm_operands(dtype=BF16):
    d = gemm_desc(8, 64, 16)
    return d, [torch.zeros(n, dtype=dtype, device="cuda") for n in (8 * 16, 16 * 64, 8 * 64, 8 * 64)]


def calls(dtype=BF16, ws=None):
    """The three operators that take a workspace, as functions of (dtype of the matrices, workspace)."""
    d, (a, b, c, z) = gemm_operands(dtype)
    m = ccl.MoeDesc(2, 4, 2, 64, 32)
    x, wr, gu, dn = (torch.zeros(n, dtype=dtype, device="cuda") for n in (2 * 64, 4 * 64, 4 * 64 * 64, 4 * 64 * 32))
    return [lambda: ccl.ccl_gemm_epilogue(d, a, b, c, ws), lambda: ccl.ccl_gemm_act_grad(d, a, b, z, c, ws, act=ccl.ACT_SILU, dbias=torch.zeros(64, dtype=BF16, device="cuda")),
            lambda: ccl.ccl_moe_tokens(m, x, wr, gu, dn, torch.zeros_like(x), ws)]


@pytest.mark.gpu
def test_workspaces_the_gpu_cannot_use():
    big = 1 << 22
    for ws in (torch.zeros(big, dtype=torch.uint8), torch.zeros(big, 2, dtype=torch.uint8, device="cuda")[:, 0]):
        for call in calls(ws=ws):
            with pytest.raises(ValueError):
                call()
    for call in calls(ws=torch.zeros(big, dtype=torch.uint8, device="cuda")):
        call()
    assert ccl.ccl_gemm_status()[0] == ccl.OK


@pytest.mark.gpu
def test_operands_left_out_are_the_librarys_to_refuse():
    d, (a, b, c, z) = gemm_operands()
    for args in ((None, b, c), (a, None, c), (a, b, None)):
        with pytest.raises(ccl.CclError) as e:
            ccl.ccl_gemm_epilogue(d, *args)
        assert e.value.status == ccl.ERR_INVALID_ARG


@pytest.mark.gpu
def test_matrices_of_another_floating_type():
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    for dtype in (torch.float16, torch.float32, torch.float64):
        for call in calls(dtype, ws):
            with pytest.raises(ValueError, match="not bfloat16"):
                call()
        g = torch.zeros(16, 8, dtype=dtype, device="cuda")
        with pytest.raises(ValueError, match="not bfloat16"):
            ccl.ccl_bias_act_grad(ccl.Mat(16, 8, 2), g, None, g)
    for call in calls(torch.int16, ws):                       # raw storage
        call()
    assert ccl.ccl_gemm_status()[0] == ccl.OK
