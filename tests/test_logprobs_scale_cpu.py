"""Scales whose product with log2(e) is no fp32 number are refused before anything is launched: exponents have the base 2, and the largest logit's
would be 0 times infinity."""
import pytest
import torch

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding

P = 1 << 20                    # an aligned address that no call may reach
LAST = 2.0 ** 127


def _forward(scale, rows):
    return rl.load_library().rlkv_token_logprobs(P, 1000, rows, 1000, rl.RLKV_F32, scale, P, P, P, P, 0, None, None, None, 0, None)


def _grad(scale, rows):
    return rl.load_library().rlkv_token_logprobs_grad(P, 1000, rows, 1000, rl.RLKV_F32, scale, P, P, P, P, P, P, 1000, None)


@pytest.mark.parametrize("call", [_forward, _grad])
def test_scale(call):
    for scale in (3.0e38, float(torch.finfo(torch.float32).max), LAST * (1 + 2.0 ** -23)):
        assert call(scale, 3) == call(scale, 0) == binding.RLKV_ERR_INVALID_ARG
    for scale in (LAST, 1e-45, 1.0):
        assert call(scale, 0) == binding.RLKV_OK          # (no rows: nothing is launched)
