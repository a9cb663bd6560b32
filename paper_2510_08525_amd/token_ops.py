"""The token-wise operators on tensors: argument checks and marshalling around the calls of include/rlkv.h.

Outputs are the caller's tensors; every call goes to the current stream of the tensors' device and returns its outputs.
Matrices are two-dimensional with contiguous columns, rows at any stride.
"""
from __future__ import annotations

import torch

from .binding import RLKV_BF16, RLKV_E4M3, RLKV_F32, _check, load_library

E4M3 = torch.float8_e4m3fn
GROUP = 128                     # columns that share a scale
_DTYPES = {torch.float32: RLKV_F32, torch.bfloat16: RLKV_BF16, E4M3: RLKV_E4M3}
_fn: dict = {}


def _call(name: str, device, *args):
    """Calls the library on the tensors' device and its current stream."""
    fn = _fn.get(name)
    if fn is None:
        fn = _fn[name] = getattr(load_library(), name)
    index = device.index
    if index == torch._C._cuda_getDevice():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status:
        _check(status, name)


def _matrix(t, what: str, device=None, dtypes=None, shape=None):
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what}: need a matrix with contiguous columns")
    return _checked(t, what, device, dtypes, shape)


def _vector(t, what: str, device=None, dtypes=None, size=None):
    if t.dim() != 1 or (t.stride(0) != 1 and t.shape[0] > 1):
        raise ValueError(f"{what}: need a contiguous vector")
    return _checked(t, what, device, dtypes, None if size is None else (size,))


def _checked(t, what, device, dtypes, shape):
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{what}: need a tensor on {device if device is not None else 'the GPU'}")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{what}: type {t.dtype} is not one of {', '.join(map(str, dtypes))}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)} != {tuple(shape)}")
    return t.data_ptr()


def groups(cols: int) -> int:
    """Groups of columns that share a scale."""
    return -(-cols // GROUP)


def rms_norm(x, weight, eps: float, out, *, scales=None, residual=None, sum_out=None):
    """out = h / sqrt(mean(h^2) + eps) * weight of h = x + residual, and sum_out = h (rlkv_rms_norm).

    `out` has the type of x, or is float8_e4m3fn: then scales [groups(cols), rows] (fp32) takes the scale of each 128 columns.
    weight, residual and sum_out may be None."""
    kinds, device = (torch.float32, torch.bfloat16), x.device
    xp = _matrix(x, "x", None, kinds)
    rows, cols = x.shape
    same = (x.dtype,)
    rp = sp = gp = wp = None
    r_stride = s_stride = g_stride = 0
    if residual is not None:
        rp, r_stride = _matrix(residual, "residual", device, same, (rows, cols)), residual.stride(0)
    if sum_out is not None:
        sp, s_stride = _matrix(sum_out, "sum_out", device, same, (rows, cols)), sum_out.stride(0)
    if weight is not None:
        wp = _vector(weight, "weight", device, same, cols)
    if scales is not None:
        gp, g_stride = _matrix(scales, "scales", device, (torch.float32,), (groups(cols), rows)), scales.stride(0)
    op = _matrix(out, "out", device, (x.dtype, E4M3), (rows, cols))
    _call("rlkv_rms_norm", device, xp, x.stride(0), rp, r_stride, wp, eps, rows, cols, _DTYPES[x.dtype], sp, s_stride, op,
          out.stride(0), _DTYPES[out.dtype], gp, g_stride)
    return out


def quantize(x, out, scales):
    """out = round(x / scale) in 8 bits, scales [groups(cols), rows]: one for each 128 columns of a row (rlkv_quantize)."""
    device = x.device
    xp = _matrix(x, "x", None, (torch.float32, torch.bfloat16))
    rows, cols = x.shape
    op = _matrix(out, "out", device, (E4M3,), (rows, cols))
    gp = _matrix(scales, "scales", device, (torch.float32,), (groups(cols), rows))
    _call("rlkv_quantize", device, xp, x.stride(0), rows, cols, _DTYPES[x.dtype], op, out.stride(0), gp, scales.stride(0))
    return out


def scaled_matmul(a, a_scales, b, b_scales, out):
    """out [m, n] = a [m, k] @ b [n, k]^T of float8_e4m3fn matrices, a_scales [groups(k), m], b_scales [groups(n), groups(k)]
    (rlkv_scaled_matmul); out is float32 or bfloat16."""
    device, scale = a.device, (torch.float32,)
    ap = _matrix(a, "a", None, (E4M3,))
    m, k = a.shape
    bp = _matrix(b, "b", device, (E4M3,))
    n = b.shape[0]
    if b.shape[1] != k:
        raise ValueError(f"b: {b.shape[1]} columns, a has {k}")
    g = groups(k)
    sa = _matrix(a_scales, "a_scales", device, scale, (g, m))
    sb = _matrix(b_scales, "b_scales", device, scale, (groups(n), g))
    op = _matrix(out, "out", device, (torch.float32, torch.bfloat16), (m, n))
    _call("rlkv_scaled_matmul", device, ap, _row_stride(a), sa, a_scales.stride(0), bp, _row_stride(b), sb, b_scales.stride(0), m, n,
          k, op, out.stride(0), _DTYPES[out.dtype])
    return out


def _rows(t, what, device, rows, dtype=torch.float32):
    return None if t is None else _vector(t, what, device, (dtype,), rows)


def token_logprobs(logits, tokens, logprobs, *, scale: float = 1.0, entropy=None, lse=None, top=None, workspace=None):
    """Log probabilities of `tokens` (int32 [rows]) under softmax(scale * logits) into logprobs [rows], and where given entropy [rows],
    lse [rows] and top = (log probabilities, int32 tokens) [rows, k] of the k most likely tokens (rlkv_token_logprobs).

    tokens and logprobs may both be None.  workspace: a uint8 tensor of rlkv_token_logprobs_workspace(rows, vocab, k) bytes that the
    caller keeps; without one the call takes one from torch's allocator."""
    device = logits.device
    xp = _matrix(logits, "logits", None, (torch.float32, torch.bfloat16))
    rows, vocab = logits.shape
    k, vp, ip = 0, None, None
    if top is not None:
        k = top[0].shape[1] if top[0].dim() == 2 else -1
        vp = _matrix(top[0], "top log probabilities", device, (torch.float32,), (rows, k))
        ip = _matrix(top[1], "top tokens", device, (torch.int32,), (rows, k))
        if not (top[0].is_contiguous() and top[1].is_contiguous()):
            raise ValueError("top: need contiguous tensors")
    need = load_library().rlkv_token_logprobs_workspace(rows, vocab, k)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    wp = _vector(workspace, "workspace", device, (torch.uint8,))
    _call("rlkv_token_logprobs", device, xp, logits.stride(0), rows, vocab, _DTYPES[logits.dtype], scale,
          _rows(tokens, "tokens", device, rows, torch.int32), _rows(logprobs, "logprobs", device, rows),
          _rows(entropy, "entropy", device, rows), _rows(lse, "lse", device, rows), k, ip, vp, wp, workspace.numel())
    return logprobs


def token_logprobs_grad(logits, tokens, lse, grad_logprobs, grad_logits, *, scale: float = 1.0, entropy=None, grad_entropy=None):
    """Gradient with respect to the logits, from the gradients of log probabilities and (where given) entropies; lse and entropy as
    token_logprobs left them (rlkv_token_logprobs_grad).  grad_logits may be logits."""
    device = logits.device
    xp = _matrix(logits, "logits", None, (torch.float32, torch.bfloat16))
    rows, vocab = logits.shape
    op = _matrix(grad_logits, "grad_logits", device, (logits.dtype,), (rows, vocab))
    _call("rlkv_token_logprobs_grad", device, xp, logits.stride(0), rows, vocab, _DTYPES[logits.dtype], scale,
          _rows(tokens, "tokens", device, rows, torch.int32), _rows(lse, "lse", device, rows), _rows(entropy, "entropy", device, rows),
          _rows(grad_logprobs, "grad_logprobs", device, rows), _rows(grad_entropy, "grad_entropy", device, rows), op,
          grad_logits.stride(0))
    return grad_logits


def _row_stride(t) -> int:
    """Distance of two rows; that of a single row, which a tensor may report as anything, is its length."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]
