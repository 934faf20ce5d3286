"""ffn.AdamW takes states of 32 or 8 bits and nothing else.  No GPU."""
import pytest

from paper_2606_11718_b200 import ffn


@pytest.mark.parametrize("bits", [16, 64, 0, 4])
def test_other_widths_are_refused(bits):
    with pytest.raises(ValueError, match="32 or 8"):
        ffn.AdamW({}, bits=bits)
