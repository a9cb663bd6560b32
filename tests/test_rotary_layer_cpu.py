"""A layer that 32 bits do not hold is refused, not taken as the one that its lower bits name."""
import pytest
import torch

import paper_2510_08525_amd as rl


@pytest.mark.parametrize("layer", [1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 31, -(1 << 31) - 1, 1 << 70])
def test_layer(layer):
    calls, shape, x = rl.tensor_calls(), (0, rl.RLKV_F32, 4, 2, 1, 64), torch.zeros(4, 1, 256)
    for call in (lambda: calls.append_rotary(0, layer, shape, x, None, 0, None), lambda: calls.rotary(0, layer, shape, x, None, 0, x, x, x)):
        with pytest.raises(ValueError, match="layer"):
            call()
