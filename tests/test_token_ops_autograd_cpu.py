"""The operators' calls are none that autograd sees: while gradients are recorded, a tensor that asks for one is refused, by its name and
before anything else is said about it (so without a GPU too)."""
import pytest
import torch

import paper_2510_08525_amd as rl


NAMES = ["rms_norm", "quantize", "scaled_matmul", "token_logprobs", "token_logprobs_grad", "append_rotary", "rotary"]


def _calls():
    x, w, v = torch.zeros(4, 256, requires_grad=True), torch.zeros(256), torch.zeros(4)
    plain = torch.zeros(4, 256)
    calls, shape = rl.tensor_calls(), (0, rl.RLKV_F32, 4, 2, 1, 64)
    return {
        "rms_norm": lambda: rl.rms_norm(x, w, 1e-5, plain),
        "quantize": lambda: rl.quantize(x * 2, plain, plain),
        "scaled_matmul": lambda: rl.scaled_matmul(x, plain, plain, plain, plain),
        "token_logprobs": lambda: rl.token_logprobs(x, None, None, lse=v, workspace=v),
        "token_logprobs_grad": lambda: rl.token_logprobs_grad(x, v, v, v, plain),
        "append_rotary": lambda: calls.append_rotary(0, 0, shape, x, None, 0, None),
        "rotary": lambda: calls.rotary(0, 0, shape, x, None, 0, plain, plain, plain),
    }


@pytest.mark.parametrize("name", NAMES)
def test_what_requires_a_gradient_is_refused(name):
    with pytest.raises(ValueError, match="requires a gradient"):
        _calls()[name]()


@pytest.mark.parametrize("name", NAMES)
def test_where_no_gradients_are_recorded_it_is_not(name):
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            with pytest.raises(ValueError, match="on the GPU|on cuda"):
                _calls()[name]()
