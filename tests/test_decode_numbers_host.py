"""A linear layer's numbers that an int does not hold are refused before its tensors are looked at (no GPU)."""
import pytest
import torch

from paper_2309_04875_amd import hb


@pytest.mark.parametrize("group,frac", [((1 << 32) + 32, 16), (32, (1 << 32) + 16), (32 - (1 << 32), 16), (32, 1 << 31), (1 << 70, 16)])
def test_numbers_out_of_range(group, frac):
    x = torch.zeros((2, 32), dtype=torch.int64)
    with pytest.raises(ValueError, match="out of range"):
        hb.hb_linear_q4(x, x, torch.zeros((16, 16), dtype=torch.uint8), torch.zeros((16, 1), dtype=torch.int32), group, frac, 7)
