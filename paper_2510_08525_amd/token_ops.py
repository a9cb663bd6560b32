"""The token-wise operators on tensors: argument checks and marshalling around the calls of include/rlkv.h.

Outputs are the caller's tensors; every call goes to the current stream of the tensors' device and returns its outputs.
Matrices are two-dimensional with contiguous columns, rows at any stride.  (A decode step makes these calls one after the other, each
of a few microseconds on the GPU: a tensor is looked at once, in one condition, and what is wrong with it is found out afterwards.)
"""
from __future__ import annotations

import torch

from .binding import RLKV_BF16, RLKV_E4M3, RLKV_F32, _check, load_library

E4M3 = torch.float8_e4m3fn
GROUP = 128                     # columns that share a scale
_F32, _I32 = torch.float32, torch.int32
_KINDS = {torch.float32: RLKV_F32, torch.bfloat16: RLKV_BF16}         # of activations and logits
_DTYPES = {**_KINDS, E4M3: RLKV_E4M3}
_current_device, _raw_stream = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)
_fn: dict = {}


def _call(name: str, index: int, *args):
    """Calls the library on the tensors' device and its current stream."""
    fn = _fn.get(name)
    if fn is None:
        fn = _fn[name] = getattr(load_library(), name)
    if index == _current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status:
        _check(status, name)


def _refuse(t, what, index, dtypes, shape):
    dtypes = dtypes if isinstance(dtypes, tuple) else (dtypes,)
    if index is not None and t.get_device() != index:
        raise ValueError(f"{what}: need a tensor on {'the GPU' if index < 0 else f'cuda:{index}'}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what}: type {t.dtype} is not one of {', '.join(map(str, dtypes))}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)} != {tuple(shape)}")
    raise ValueError(f"{what}: need a {'contiguous vector' if t.dim() == 1 else 'matrix with contiguous columns'}")


def _first(t, what):
    """The matrix a call is about: (address, row stride, rows, columns, device, kind)."""
    index, kind = t.get_device(), _KINDS.get(t.dtype)
    if kind is None or index < 0 or t.dim() != 2:
        _refuse(t, what, -2 if index < 0 else None, tuple(_KINDS), None)
    rows, cols = t.shape
    stride = t.stride()
    if stride[1] != 1 and cols > 1:
        _refuse(t, what, None, tuple(_KINDS), None)
    return t.data_ptr(), stride[0], rows, cols, index, kind


def _matrix(t, what, index, dtype, shape):
    """(address, row stride) of a matrix of this type and shape."""
    stride = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or (stride[1] != 1 and shape[1] > 1):
        _refuse(t, what, index, dtype, shape)
    return t.data_ptr(), stride[0]


def _vector(t, what, index, dtype, size):
    """Address of a vector of this type and size; None of None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != (size,) or t.get_device() != index or (size > 1 and t.stride(0) != 1):
        _refuse(t, what, index, dtype, (size,))
    return t.data_ptr()


def groups(cols: int) -> int:
    """Groups of columns that share a scale."""
    return -(-cols // GROUP)


def rms_norm(x, weight, eps: float, out, *, scales=None, residual=None, sum_out=None):
    """out = h / sqrt(mean(h^2) + eps) * weight of h = x + residual, and sum_out = h (rlkv_rms_norm).

    `out` has the type of x, or is float8_e4m3fn: then scales [groups(cols), rows] (fp32) takes the scale of each 128 columns.
    weight, residual and sum_out may be None."""
    xp, x_stride, rows, cols, index, kind = _first(x, "x")
    dtype, shape = x.dtype, (rows, cols)
    rp = sp = gp = None
    r_stride = s_stride = g_stride = 0
    if residual is not None:
        rp, r_stride = _matrix(residual, "residual", index, dtype, shape)
    if sum_out is not None:
        sp, s_stride = _matrix(sum_out, "sum_out", index, dtype, shape)
    if scales is not None:
        gp, g_stride = _matrix(scales, "scales", index, _F32, (-(-cols // GROUP), rows))
    wp = _vector(weight, "weight", index, dtype, cols)
    out_kind = RLKV_E4M3 if out.dtype is E4M3 else kind
    op, o_stride = _matrix(out, "out", index, E4M3 if out_kind == RLKV_E4M3 else dtype, shape)
    _call("rlkv_rms_norm", index, xp, x_stride, rp, r_stride, wp, eps, rows, cols, kind, sp, s_stride, op, o_stride, out_kind, gp, g_stride)
    return out


def quantize(x, out, scales):
    """out = round(x / scale) in 8 bits, scales [groups(cols), rows]: one for each 128 columns of a row (rlkv_quantize)."""
    xp, x_stride, rows, cols, index, kind = _first(x, "x")
    op, o_stride = _matrix(out, "out", index, E4M3, (rows, cols))
    gp, g_stride = _matrix(scales, "scales", index, _F32, (-(-cols // GROUP), rows))
    _call("rlkv_quantize", index, xp, x_stride, rows, cols, kind, op, o_stride, gp, g_stride)
    return out


def scaled_matmul(a, a_scales, b, b_scales, out):
    """out [m, n] = a [m, k] @ b [n, k]^T of float8_e4m3fn matrices, a_scales [groups(k), m], b_scales [groups(n), groups(k)]
    (rlkv_scaled_matmul); out is float32 or bfloat16."""
    index, kind = a.get_device(), _KINDS.get(out.dtype)
    if index < 0 or a.dim() != 2 or b.dim() != 2:
        raise ValueError("a, b: need matrices on the GPU")
    if kind is None:
        _refuse(out, "out", None, tuple(_KINDS), None)
    m, k = a.shape
    n = b.shape[0]
    g = -(-k // GROUP)
    ap, a_stride = _matrix(a, "a", index, E4M3, (m, k))
    bp, b_stride = _matrix(b, "b", index, E4M3, (n, k))
    sa, sa_stride = _matrix(a_scales, "a_scales", index, _F32, (g, m))
    sb, sb_stride = _matrix(b_scales, "b_scales", index, _F32, (-(-n // GROUP), g))
    op, o_stride = _matrix(out, "out", index, out.dtype, (m, n))
    # (the distance of two rows of a matrix with one, which a tensor may report as anything, is its length)
    _call("rlkv_scaled_matmul", index, ap, a_stride if m > 1 else k, sa, sa_stride, bp, b_stride if n > 1 else k, sb, sb_stride, m, n, k,
          op, o_stride if m > 1 else n, kind)
    return out


def token_logprobs(logits, tokens, logprobs, *, scale: float = 1.0, entropy=None, lse=None, top=None, workspace=None):
    """Log probabilities of `tokens` (int32 [rows]) under softmax(scale * logits) into logprobs [rows], and where given entropy [rows],
    lse [rows] and top = (log probabilities, int32 tokens) [rows, k] of the k most likely tokens (rlkv_token_logprobs).

    tokens and logprobs may both be None.  workspace: a uint8 tensor of rlkv_token_logprobs_workspace(rows, vocab, k) bytes that the
    caller keeps; without one the call takes one from torch's allocator."""
    xp, stride, rows, vocab, index, kind = _first(logits, "logits")
    k, vp, ip = 0, None, None
    if top is not None:
        k = top[0].shape[1] if top[0].dim() == 2 else -1
        vp, v_stride = _matrix(top[0], "top log probabilities", index, _F32, (rows, k))
        ip, i_stride = _matrix(top[1], "top tokens", index, _I32, (rows, k))
        if rows > 1 and (v_stride != k or i_stride != k):
            raise ValueError("top: need contiguous tensors")
    if workspace is None:
        need = load_library().rlkv_token_logprobs_workspace(rows, vocab, k)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=logits.device)
    room = workspace.numel()
    _call("rlkv_token_logprobs", index, xp, stride, rows, vocab, kind, scale, _vector(tokens, "tokens", index, _I32, rows),
          _vector(logprobs, "logprobs", index, _F32, rows), _vector(entropy, "entropy", index, _F32, rows),
          _vector(lse, "lse", index, _F32, rows), k, ip, vp, _vector(workspace, "workspace", index, torch.uint8, room), room)
    return logprobs


def token_logprobs_grad(logits, tokens, lse, grad_logprobs, grad_logits, *, scale: float = 1.0, entropy=None, grad_entropy=None):
    """Gradient with respect to the logits, from the gradients of log probabilities and (where given) entropies; lse and entropy as
    token_logprobs left them (rlkv_token_logprobs_grad).  grad_logits may be logits."""
    xp, stride, rows, vocab, index, kind = _first(logits, "logits")
    op, o_stride = _matrix(grad_logits, "grad_logits", index, logits.dtype, (rows, vocab))
    _call("rlkv_token_logprobs_grad", index, xp, stride, rows, vocab, kind, scale, _vector(tokens, "tokens", index, _I32, rows),
          _vector(lse, "lse", index, _F32, rows), _vector(entropy, "entropy", index, _F32, rows),
          _vector(grad_logprobs, "grad_logprobs", index, _F32, rows), _vector(grad_entropy, "grad_entropy", index, _F32, rows), op, o_stride)
    return grad_logits
