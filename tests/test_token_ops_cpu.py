"""Refusals of the token-wise operators: every check runs on the host before the first HIP call."""
import pytest

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


def test_the_package_offers_them():
    for name in ("rms_norm", "quantize"):
        assert callable(getattr(rl, name))
    with pytest.raises(AttributeError):
        rl.no_such_operator
