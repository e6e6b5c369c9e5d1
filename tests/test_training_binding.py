"""The Python names of the training operators: what they refuse before the library is called (no GPU)."""
import pytest
import torch

from paper_2208_09151_amd import training


def test_restore_refuses_codes_that_are_not_on_the_current_gpu():
    """Without `out` nothing else of the call is in the current GPU's memory."""
    there = training.Compressed._made(torch.zeros((3, 64), dtype=torch.int8), torch.zeros((3, 2), dtype=torch.uint8), 64)
    with pytest.raises(ValueError, match="kept"):
        training.restore(there)


@pytest.mark.parametrize("slots, width, out", [(16, 4096, 4096), (64, 65_536, 65_536), (100, 3000, 1 << 20)])
def test_a_weight_gradient_in_one_range_needs_no_room_for_parts(slots, width, out):
    """Few slots of wide layers: the tiles alone fill the GPU, and no expert is shared by ranges."""
    lib = training._lib.load()
    assert 0 < lib.ginex_weight_gradient_workspace_bytes(slots, 1, width, out) <= 4096
    # many slots of a narrow one: two parts a range at most
    assert lib.ginex_weight_gradient_workspace_bytes(1_000_000, 4, 64, 64) <= 2 * 512 * 64 * 64 * 4 + 4096
