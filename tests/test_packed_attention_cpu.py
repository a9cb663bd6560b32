"""Refusals of the attention over packed sequences: every check runs on the host before the first HIP call."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding

BAD, OK = binding.RLKV_ERR_INVALID_ARG, binding.RLKV_OK
P = 1 << 20                    # an aligned address that no call may reach
MASK = np.array([1, 0], dtype=np.uint8)


def _call(grad=False, **over):
    a = dict(offsets=P, n_seqs=3, tokens=100, n_q_heads=8, n_kv_heads=2, full_mask=MASK.ctypes.data, sink=4, recent=60, softmax_scale=0.1, lse=P,
             workspace=P, workspace_bytes=1 << 20)
    heads = dict(q=8, k=2, v=2, out=8)
    if grad:
        heads.update(grad_out=8, grad_q=8, grad_k=2, grad_v=2)
    for name, h in heads.items():
        a[name] = (P, h * 128, 128)
    a.update(over)
    shape = binding.Packed(*(a[f] for f, _ in binding.Packed._fields_))
    p = {n: ctypes.byref(binding.Heads(*a[n])) if a[n] is not None else None for n in heads}
    lib = rl.load_library()
    if not grad:
        return lib.rlkv_packed_attention(ctypes.byref(shape), p["q"], p["k"], p["v"], p["out"], a["lse"], None)
    return lib.rlkv_packed_attention_grad(ctypes.byref(shape), p["q"], p["k"], p["v"], p["out"], a["lse"], p["grad_out"], p["grad_q"],
                                          p["grad_k"], p["grad_v"], a["workspace"], a["workspace_bytes"], None)


TWO = np.array([1, 2], dtype=np.uint8)
SHAPES = [dict(offsets=None), dict(offsets=P + 2), dict(n_seqs=-1), dict(n_seqs=2 ** 31 - 1), dict(tokens=-1), dict(tokens=2 ** 28), dict(n_q_heads=0),
          dict(n_q_heads=9), dict(n_kv_heads=0), dict(n_q_heads=34), dict(n_q_heads=514, n_kv_heads=257, full_mask=None), dict(sink=-1),
          dict(recent=0), dict(recent=-1), dict(full_mask=TWO.ctypes.data), dict(softmax_scale=0.0), dict(softmax_scale=-1.0),
          dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(lse=P + 2)]
ROWS = [None, (None, 1024, 128), (P + 8, 1024, 128), (P, 1028, 128), (P, 1024, 132), (P, -1024, 128), (P, 1024, -128), (P, 2 ** 41, 128)]
WRITTEN = [(P, 0, 128), (P, 1016, 128), (P, 1024, 120), (P, 128, 128)]


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("bad", SHAPES)
def test_shapes_are_refused(bad, grad):
    assert _call(grad, **bad) == BAD


@pytest.mark.parametrize("name", ["q", "k", "v", "out", "grad_out", "grad_q", "grad_k", "grad_v"])
@pytest.mark.parametrize("row", ROWS)
def test_rows_are_refused(name, row):
    assert _call(True, **{name: row}) == BAD
    if not name.startswith("grad"):
        assert _call(False, **{name: row}) == BAD


@pytest.mark.parametrize("name", ["out", "grad_q"])
@pytest.mark.parametrize("row", WRITTEN)
def test_outputs_whose_rows_overlap_are_refused(name, row):
    assert _call(name != "out", **{name: row}) == BAD


@pytest.mark.parametrize("bad", [dict(workspace=None), dict(workspace=P + 8), dict(workspace_bytes=100), dict(lse=None)])
def test_the_gradient_refuses(bad):
    assert _call(True, **bad) == BAD


def test_nothing_to_do():
    nothing = dict(q=None, k=None, v=None, out=None, offsets=None, lse=None)
    assert _call(tokens=0, **nothing) == OK and _call(n_seqs=0, **nothing) == OK
    nothing.update(grad_out=None, grad_q=None, grad_k=None, grad_v=None, workspace=None, workspace_bytes=0)
    assert _call(True, tokens=0, **nothing) == OK and _call(True, n_seqs=0, **nothing) == OK


def test_workspace():
    need = rl.rlkv_packed_attention_grad_workspace
    assert need(0, 8, 2) == need(-1, 8, 2) == need(10, 8, 3) == need(10, 0, 1) == need(10, 34, 2) == need(2 ** 29, 8, 2) == 0
    assert need(1, 1, 1) > 0 and need(1000, 8, 2) >= 32000


def test_what_is_no_tensor_of_a_device_is_refused():
    x, o = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for f in (lambda: rl.packed_attention(x, x, x, o, x, 0.1), lambda: rl.packed_attention(1, x, x, o, x, 0.1),
              lambda: rl.packed_attention_grad(x, x, x, o, x, x, x, x, x, x, 0.1)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        rl.tensor_calls().packed_attention(x, x)
