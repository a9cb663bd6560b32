"""Refusals of the token-wise operators: every check runs on the host before the first HIP call."""
import pytest
import torch

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding

BAD, OK = binding.RLKV_ERR_INVALID_ARG, binding.RLKV_OK
P = 1 << 20                    # an aligned address that no call may reach


def _norm(**over):
    a = dict(x=P, x_stride=256, residual=P, residual_stride=256, weight=P, eps=1e-5, rows=4, cols=256, dtype=rl.RLKV_BF16, sum_out=P,
             sum_stride=256, out=P, out_stride=256, out_dtype=rl.RLKV_E4M3, scales=P, scale_stride=4)
    a.update(over)
    return rl.load_library().rlkv_rms_norm(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(out=None), dict(rows=-1), dict(cols=0), dict(cols=-5), dict(dtype=2), dict(dtype=7), dict(out_dtype=0),
    dict(out_dtype=9), dict(x_stride=-256), dict(out_stride=255), dict(sum_stride=255), dict(residual=None), dict(residual_stride=-1),
    dict(scales=None), dict(scale_stride=3), dict(out_dtype=1), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(x=P + 1), dict(residual=P + 1), dict(weight=P + 1), dict(scales=P + 2), dict(sum_out=P + 1),
    dict(dtype=0, x=P + 2), dict(dtype=0, out_dtype=1),
])
def test_norm_refuses(bad):
    assert _norm(**bad) == BAD


def test_norm_without_rows():
    assert _norm(rows=0) == OK


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(out=None), dict(scales=None), dict(rows=-2), dict(cols=0), dict(dtype=2), dict(x_stride=-1), dict(out_stride=100),
    dict(scale_stride=2), dict(x=P + 1), dict(scales=P + 1),
])
def test_quantize_refuses(bad):
    a = dict(x=P, x_stride=300, rows=3, cols=300, dtype=rl.RLKV_BF16, out=P, out_stride=300, scales=P, scale_stride=3)
    a.update(bad)
    assert rl.load_library().rlkv_quantize(*a.values(), None) == BAD


@pytest.mark.parametrize("bad", [
    dict(a=None), dict(b=None), dict(a_scales=None), dict(b_scales=None), dict(out=None), dict(m=-1), dict(n=-1), dict(k=0), dict(k=-128),
    dict(k=250), dict(k=8), dict(out_dtype=2), dict(out_dtype=5), dict(a=P + 8), dict(b=P + 4), dict(a_stride=264), dict(b_stride=250),
    dict(a_stride=-256), dict(b_stride=-16), dict(a_stride=(1 << 23) + 16), dict(b_stride=(1 << 23) + 16), dict(out_stride=299),
    dict(a_scale_stride=-1), dict(b_scale_stride=-1), dict(a_scales=P + 1), dict(out=P + 1), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 1),
    dict(k=(1 << 24) + 16), dict(m=1 << 24, n=1 << 24, out_stride=1 << 24), dict(out_dtype=0, out=P + 2),
])
def test_matmul_refuses(bad):
    a = dict(a=P, a_stride=256, a_scales=P, a_scale_stride=5, b=P, b_stride=256, b_scales=P, b_scale_stride=2, m=5, n=300, k=256, out=P,
             out_stride=300, out_dtype=rl.RLKV_BF16)
    a.update(bad)
    assert rl.load_library().rlkv_scaled_matmul(*a.values(), None) == BAD


def test_matmul_of_nothing():
    call = rl.load_library().rlkv_scaled_matmul
    assert call(None, 0, None, 0, P, 128, P, 1, 0, 7, 128, P, 7, 1, None) == OK
    assert call(P, 128, P, 7, None, 0, None, 0, 7, 0, 128, P, 7, 1, None) == OK


def test_the_package_offers_them():
    for name in ("rms_norm", "quantize", "scaled_matmul"):
        assert callable(getattr(rl, name))
    with pytest.raises(AttributeError):
        rl.no_such_operator


def test_rotary_without_a_cache_is_refused():
    lib, r = rl.load_library(), rl.Rotary([1.0] * 64)
    assert lib.rlkv_append_rotary(None, 0, P, 1024, None, 1, r.address, P, None) == BAD
    assert lib.rlkv_rotary(None, 0, P, 1024, None, 1, r.address, P, P, P, None) == BAD


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dtype=2), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(stride=-1), dict(logits=P + 1), dict(tokens=None),
    dict(logprobs=None), dict(top=-1), dict(top=33), dict(top=20, vocab=19), dict(top_ids=None), dict(top_logprobs=None), dict(tokens=P + 2),
    dict(entropy=P + 1), dict(lse=P + 1), dict(top_ids=P + 2), dict(workspace=None), dict(workspace=P + 4), dict(workspace_bytes=100),
])
def test_logprobs_refuse(bad):
    a = dict(logits=P, stride=50000, rows=3, vocab=50000, dtype=rl.RLKV_BF16, scale=1.0, tokens=P, logprobs=P, entropy=P, lse=P, top=5,
             top_ids=P, top_logprobs=P, workspace=P, workspace_bytes=1 << 20)
    a.update(bad)
    assert rl.load_library().rlkv_token_logprobs(*a.values(), None) == BAD


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(rows=-1), dict(vocab=0), dict(dtype=2), dict(scale=0.0), dict(tokens=None), dict(lse=None), dict(entropy=None),
    dict(grad_logprobs=None), dict(grad_entropy=None), dict(grad_logits=None), dict(grad_stride=999), dict(stride=-1), dict(lse=P + 1),
    dict(grad_logits=P + 1),
])
def test_logprobs_grad_refuses(bad):
    a = dict(logits=P, stride=1000, rows=3, vocab=1000, dtype=rl.RLKV_BF16, scale=1.0, tokens=P, lse=P, entropy=P, grad_logprobs=P,
             grad_entropy=P, grad_logits=P, grad_stride=1000)
    a.update(bad)
    assert rl.load_library().rlkv_token_logprobs_grad(*a.values(), None) == BAD


def test_logprobs_workspace():
    need = rl.rlkv_token_logprobs_workspace
    assert need(0, 100, 0) == need(4, 0, 0) == need(4, 100, 33) == need(4, 100, -1) == need(-1, 100, 0) == 0
    assert need(5000, 100000, 20) == 0 and need(1, 16384, 32) == 0            # nothing is split
    assert 0 < need(2, 100000, 0) < need(2, 100000, 20)


def test_what_is_no_tensor_of_a_device_is_refused():
    x = torch.zeros(4, 256)
    v = torch.zeros(4)
    calls = rl.tensor_calls()
    shape = (0, rl.RLKV_F32, 4, 2, 1, 64)
    for f in (lambda: rl.rms_norm(x, None, 1e-5, x), lambda: rl.quantize(x, x, x), lambda: rl.scaled_matmul(x, x, x, x, x),
              lambda: rl.token_logprobs(x, None, None, lse=v, workspace=v), lambda: rl.token_logprobs_grad(x, v, v, v, x),
              lambda: rl.quantize(3, x, x), lambda: rl.rms_norm(None, None, 1e-5, x),
              lambda: calls.append_rotary(0, 0, shape, x, None, 0, None), lambda: calls.rotary(None, 0, shape, 1, None, 0, x, x, x)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: calls.quantize(x, x), lambda: calls.append_rotary(0, 0, shape[:5], x, None, 0, None),
              lambda: calls.append_rotary(0, "0", shape, x, None, 0, None)):
        with pytest.raises(TypeError):
            f()


@pytest.mark.parametrize("cols", [(1 << 30) + 1, (1 << 31) - 1])
def test_rows_longer_than_the_indexes_are_refused(cols):
    assert _norm(cols=cols, x_stride=cols, residual_stride=cols, sum_stride=cols, out_stride=cols) == BAD


@pytest.mark.parametrize("m, n", [(1 << 18, 1 << 18), (1 << 24, 1 << 13), (1 << 12, 1 << 24)])
def test_products_of_more_threads_than_a_launch_has_are_refused(m, n):
    call = rl.load_library().rlkv_scaled_matmul
    assert call(P, 128, P, m, P, 128, P, 1, m, n, 128, P, n, rl.RLKV_BF16, None) == BAD
