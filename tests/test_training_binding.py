"""The Python names of the training operators: what they refuse before the library is called (no GPU)."""
import pytest
import torch

from paper_2208_09151_amd import training


def test_restore_refuses_codes_that_are_not_on_the_current_gpu():
    """Without `out` nothing else of the call is in the current GPU's memory."""
    there = training.Compressed._made(torch.zeros((3, 64), dtype=torch.int8), torch.zeros((3, 2), dtype=torch.uint8), 64)
    with pytest.raises(ValueError, match="kept"):
        training.restore(there)
