"""The types of a gathered output that are refused before any device work."""
import types

import pytest
import torch

from paper_2511_12500_amd import heap


@pytest.mark.parametrize("dtype", [torch.float32, torch.float64, torch.uint8, torch.int16])
def test_outputs_are_of_16_bit_floating_point(dtype):
    """Results are stored as one of the two 16-bit types: as any other they would be read wrong,
    and behind their end."""
    with pytest.raises(TypeError, match="float16 or bfloat16"):
        heap.GatheredOutput(types.SimpleNamespace(world=2), 4, 16, dtype, 64, 16)
