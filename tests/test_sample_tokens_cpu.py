"""Refusals of the drawing of tokens: every check runs on the host before the first HIP call."""
import ctypes

import pytest
import torch

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding

BAD, OK = binding.RLKV_ERR_INVALID_ARG, binding.RLKV_OK
P = 1 << 20


def call(**over):
    how = dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0, temperatures=None, top_ps=None, min_ps=None, top_ks=None)
    a = dict(logits=P, stride=1000, rows=3, vocab=1000, dtype=rl.RLKV_BF16, how=how, uniforms=P, tokens=P, logprobs=P, workspace=P, workspace_bytes=1 << 24)
    for k, v in over.items():
        (how if k in how else a)[k] = v
    if a["how"] is not None:
        s = binding.Sampling(**how)
        a["how"] = ctypes.addressof(s)
    return rl.load_library().rlkv_sample_tokens(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(logits=P + 1), dict(stride=-1), dict(stride=2 ** 41), dict(rows=-1), dict(rows=2 ** 20 + 1), dict(vocab=0), dict(vocab=2 ** 24 + 1),
    dict(dtype=2), dict(how=None), dict(uniforms=None), dict(uniforms=P + 2), dict(tokens=None), dict(tokens=P + 2), dict(logprobs=P + 2),
    dict(temperature=-0.1), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=-0.1), dict(top_p=float("nan")),
    dict(min_p=-0.1), dict(min_p=1.1), dict(min_p=float("nan")), dict(temperatures=P + 2), dict(top_ks=P + 2), dict(top_ps=P + 2), dict(min_ps=P + 2),
    dict(dtype=0, logits=P + 2)])
def test_refuses(bad):
    assert call(**bad) == BAD


def test_nothing_to_do():
    assert call(rows=0, logits=None, uniforms=None, tokens=None, logprobs=None, workspace=None) == OK


def test_workspace():
    need = rl.rlkv_sample_tokens_workspace
    assert need(0, 100) == need(-1, 100) == need(3, 0) == need(2 ** 20 + 1, 10) == need(3, 2 ** 24 + 1) == 0


def test_what_is_no_tensor_of_a_device_is_refused():
    x, u, t = torch.zeros(4, 50), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for f in (lambda: rl.sample_tokens(x, u, t), lambda: rl.tensor_calls().sample_tokens(1, u, t, 1.0, 0, 1.0, 0.0, None, u)):
        with pytest.raises(ValueError):
            f()
