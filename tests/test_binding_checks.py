"""What the binding refuses before a call reaches the library.  No GPU is needed."""
import pytest
import torch

from paper_2607_23264_b200 import binding


def test_the_gain_is_known_by_its_type():
    assert binding._gain_fp32(torch.ones(8, dtype=torch.bfloat16)) == 0
    assert binding._gain_fp32(torch.ones(8)) == 1
    for dtype in (torch.float16, torch.int16, torch.int32, torch.float64, torch.uint8):
        with pytest.raises(ValueError, match="bf16 or fp32"):
            binding._gain_fp32(torch.ones(8, dtype=dtype))
    with pytest.raises(ValueError, match="bf16 or fp32"):
        binding._gain_fp32(None)
