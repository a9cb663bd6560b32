"""Refusals of the heads' norm with rotation and of its gradient: every check runs on the host before the first HIP call."""
import ctypes

import pytest
import torch

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding

BAD, OK = binding.RLKV_ERR_INVALID_ARG, binding.RLKV_OK
P = 1 << 20
TURN = rl.Rotary([1.0] * 64)
KEEP = []


def norm(eps, wq=P, wk=P):
    KEEP.append(binding.HeadNorm(wq, wk, eps))
    return ctypes.addressof(KEEP[-1])


def rows(h, data=P, token=None, head=128):
    KEEP.append(binding.Heads(data, h * 128 if token is None else token, head))
    return ctypes.addressof(KEEP[-1])


def forward(**over):
    a = dict(qkv=P, token_stride=1536, positions=P, rotary=TURN.address, norm=norm(1e-6), tokens=10, n_q_heads=8, n_kv_heads=2, dtype=rl.RLKV_BF16,
             q_out=rows(8), k_out=rows(2), v_out=rows(2))
    a.update(over)
    return rl.load_library().rlkv_head_norm_rotary(*a.values(), None)


def backward(**over):
    a = dict(qkv=P, token_stride=1536, positions=P, rotary=TURN.address, norm=norm(1e-6), tokens=10, n_q_heads=8, n_kv_heads=2, dtype=rl.RLKV_BF16,
             grad_q=rows(8), grad_k=rows(2), grad_v=None, grad_qkv=P, grad_stride=1536, grad_q_weight=P, grad_k_weight=P, workspace=P,
             workspace_bytes=1 << 24)
    a.update(over)
    return rl.load_library().rlkv_head_norm_rotary_grad(*a.values(), None)


BOTH = [dict(qkv=None), dict(qkv=P + 1), dict(token_stride=1535), dict(token_stride=-1536), dict(token_stride=2 ** 41), dict(positions=None),
        dict(positions=P + 2), dict(norm=norm(-1.0)), dict(norm=norm(float("nan"))), dict(norm=norm(float("inf"))), dict(norm=norm(1e-6, P + 1)),
        dict(norm=norm(1e-6, P, P + 1)), dict(tokens=-1), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=2 ** 16 + 1, token_stride=2 ** 30),
        dict(tokens=2 ** 27), dict(dtype=2), dict(dtype=7), dict(rotary=rl.Rotary([1.0] * 4).address), dict(rotary=rl.Rotary([float("inf")] * 8).address),
        dict(rotary=rl.Rotary([1.0] * 72).address)]


@pytest.mark.parametrize("bad", BOTH)
def test_both_refuse(bad):
    KEEP.append([rl.Rotary([1.0] * 4)])
    assert forward(**bad) == BAD and backward(**bad) == BAD


@pytest.mark.parametrize("bad", [dict(q_out=None), dict(k_out=None), dict(q_out=rows(8, P + 8)), dict(k_out=rows(2, token=0)), dict(v_out=rows(2, P, 255)),
                                 dict(q_out=rows(8, head=120)), dict(q_out=rows(8, token=1020))])
def test_forward_refuses(bad):
    assert forward(**bad) == BAD


@pytest.mark.parametrize("bad", [dict(grad_q=None), dict(grad_k=None), dict(grad_q=rows(8, P + 8)), dict(grad_v=rows(2, P + 4)), dict(grad_qkv=None),
                                 dict(grad_qkv=P + 1), dict(grad_stride=1535), dict(grad_stride=2 ** 41), dict(grad_q_weight=P + 2), dict(norm=None),
                                 dict(workspace=None), dict(workspace=P + 8), dict(workspace_bytes=100)])
def test_backward_refuses(bad):
    assert backward(**bad) == BAD


def test_nothing_to_do():
    assert forward(tokens=0, qkv=None, positions=None, q_out=None, k_out=None, v_out=None) == OK
    assert backward(tokens=0, qkv=None, positions=None, grad_q=None, grad_k=None, grad_qkv=None, grad_q_weight=None, grad_k_weight=None, workspace=None) == OK


def test_workspace():
    need = rl.rlkv_head_norm_rotary_grad_workspace
    assert need(0, 8, 2) == need(-1, 8, 2) == need(10, 0, 2) == need(10, 8, 0) == need(2 ** 29, 8, 2) == 0
    assert 0 < need(1, 8, 2) < need(1000, 8, 2) <= need(10 ** 6, 8, 2) < 1 << 24


def test_what_is_no_tensor_of_a_device_is_refused():
    x, p = torch.zeros(4, 512), torch.zeros(4, dtype=torch.int32)
    for f in (lambda: rl.head_norm_rotary(x, p, TURN, x.view(4, 4, 128)[:, :2], x.view(4, 4, 128)[:, 2:3]),
              lambda: rl.head_norm_rotary_grad(x, p, TURN, x.view(4, 4, 128)[:, :2], x.view(4, 4, 128)[:, 2:3], x), lambda: rl.head_norm_rotary(1, p, TURN, x, x)):
        with pytest.raises(ValueError):
            f()
