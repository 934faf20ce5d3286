"""The stream handle that every call passes on: torch's short way to it where there is one, the public one elsewhere."""
import subprocess
import sys
import types

import pytest
import torch

from paper_2606_11718_b200 import binding as ccl


@pytest.mark.parametrize("missing", ["_raw_stream", "_raw_device"])
def test_without_torchs_private_calls(monkeypatch, missing):
    monkeypatch.setattr(ccl, "_raw_stream", lambda device: 7)
    monkeypatch.setattr(ccl, "_raw_device", lambda: 0)
    assert ccl._stream() == 7
    monkeypatch.setattr(ccl, missing, None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=11))
    assert ccl._stream() == 11


@pytest.mark.gpu
def test_both_ways_give_the_same_handle():
    for s in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            assert ccl._stream() == torch.cuda.current_stream().cuda_stream == s.cuda_stream


@pytest.mark.gpu
def test_the_first_call_of_a_process():
    code = "from paper_2606_11718_b200 import binding as ccl; assert ccl.ccl_gemm_status() == (ccl.OK, 0)"
    subprocess.run([sys.executable, "-c", code], check=True, timeout=300)
