"""The token-wise operators on tensors, around the calls of include/rlkv.h (checks and marshalling: csrc/tensor_calls.cpp).

Outputs are the caller's tensors; every call goes to the current stream of the tensors' device and returns its outputs.
Matrices are two-dimensional with contiguous columns, rows at any stride.  What is wrong with a tensor raises ValueError, what the library
refuses RlkvError.  Autograd does not see the calls: as with torch's own calls into given outputs, a tensor that requires a gradient is
refused unless under torch.no_grad(), and what is written counts as changed in place (`token_logprobs_grad` is the way back).
"""
from __future__ import annotations

import torch

from .binding import _check, load_library, tensor_calls

GROUP = 128                     # columns that share a scale
_calls = tensor_calls()


def groups(cols: int) -> int:
    """Groups of columns that share a scale."""
    return -(-cols // GROUP)


def rms_norm(x, weight, eps: float, out, *, scales=None, residual=None, sum_out=None):
    """out = h / sqrt(mean(h^2) + eps) * weight of h = x + residual, and sum_out = h (rlkv_rms_norm).

    `out` has the type of x, or is float8_e4m3fn: then scales [groups(cols), rows] (fp32) takes the scale of each 128 columns.
    weight, residual and sum_out may be None."""
    status = _calls.rms_norm(x, weight, eps, out, scales, residual, sum_out)
    if status:
        _check(status, "rlkv_rms_norm")
    return out


def quantize(x, out, scales):
    """out = round(x / scale) in 8 bits, scales [groups(cols), rows]: one for each 128 columns of a row (rlkv_quantize)."""
    status = _calls.quantize(x, out, scales)
    if status:
        _check(status, "rlkv_quantize")
    return out


def scaled_matmul(a, a_scales, b, b_scales, out):
    """out [m, n] = a [m, k] @ b [n, k]^T of float8_e4m3fn matrices, a_scales [groups(k), m], b_scales [groups(n), groups(k)]
    (rlkv_scaled_matmul); out is float32 or bfloat16."""
    status = _calls.scaled_matmul(a, a_scales, b, b_scales, out)
    if status:
        _check(status, "rlkv_scaled_matmul")
    return out


def token_logprobs(logits, tokens, logprobs, *, scale: float = 1.0, entropy=None, lse=None, top=None, workspace=None):
    """Log probabilities of `tokens` (int32 [rows]) under softmax(scale * logits) into logprobs [rows], and where given entropy [rows],
    lse [rows] and top = (log probabilities, int32 tokens) [rows, k] of the k most likely tokens (rlkv_token_logprobs).

    tokens and logprobs may both be None.  workspace: a uint8 tensor of rlkv_token_logprobs_workspace(rows, vocab, k) bytes that the
    caller keeps; without one the call takes one from torch's allocator."""
    values, ids = (None, None) if top is None else top
    if workspace is None:
        rows, vocab = logits.shape if logits.dim() == 2 else (0, 0)
        k = values.shape[-1] if values is not None and values.dim() else 0
        need = load_library().rlkv_token_logprobs_workspace(rows, vocab, k)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=logits.device)
    status = _calls.token_logprobs(logits, tokens, logprobs, scale, entropy, lse, values, ids, workspace)
    if status:
        _check(status, "rlkv_token_logprobs")
    return logprobs


def token_logprobs_grad(logits, tokens, lse, grad_logprobs, grad_logits, *, scale: float = 1.0, entropy=None, grad_entropy=None):
    """Gradient with respect to the logits, from the gradients of log probabilities and (where given) entropies; lse and entropy as
    token_logprobs left them (rlkv_token_logprobs_grad).  grad_logits may be logits."""
    status = _calls.token_logprobs_grad(logits, tokens, lse, grad_logprobs, grad_logits, scale, entropy, grad_entropy)
    if status:
        _check(status, "rlkv_token_logprobs_grad")
    return grad_logits
