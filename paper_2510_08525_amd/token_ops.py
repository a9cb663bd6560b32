"""The token-wise operators and those of packed sequences on tensors, around the calls of include/rlkv.h (checks and marshalling:
csrc/tensor_calls.cpp).

Outputs are the caller's tensors; every call goes to the current stream of the tensors' device and returns its outputs.
Matrices are two-dimensional with contiguous columns, rows at any stride.  What is wrong with a tensor raises ValueError, what the library
refuses RlkvError.  Autograd does not see the calls: as with torch's own calls into given outputs, a tensor that requires a gradient is
refused unless under torch.no_grad(), and what is written counts as changed in place (`token_logprobs_grad`,
`packed_attention_grad` and `head_norm_rotary_grad` are the ways back).
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


def _mask_bytes(mask):
    """(By its entries: of a number, and of a tensor with one entry, `bytes` would take the value for a length.)"""
    if mask is None:
        return None
    try:
        return bytes(iter(mask))
    except TypeError:
        raise ValueError("mask: need a 0 or 1 for each KV head") from None


def packed_attention(q, k, v, offsets, out, scale: float, *, lse=None, mask=None, sink: int = 0, recent: int = 0):
    """Attention over sequences packed one behind the other, q and out [tokens, q heads, 128], k and v [tokens, kv heads, 128] in bfloat16
    (heads and tokens at any stride, rows at multiples of 16 bytes): out = softmax(scale * q . k) v over the keys up to the query's own, and
    lse [q heads, tokens] (float32) the log-sum-exp of the scores (rlkv_packed_attention).

    offsets: int32 [sequences + 1] on the device, where the sequences begin and the last one ends; rows of none are not written.
    mask: one 0 / 1 for each KV head, 1 = full, 0 = local (the first `sink` positions of the sequence and the last `recent`); None: all full."""
    status = _calls.packed_attention(q, k, v, offsets, out, lse, scale, _mask_bytes(mask), sink, recent)
    if status:
        _check(status, "rlkv_packed_attention")
    return out


def packed_attention_grad(q, k, v, offsets, out, lse, grad_out, grad_q, grad_k, grad_v, scale: float, *, mask=None, sink: int = 0,
                          recent: int = 0, workspace=None):
    """Gradients of packed_attention's q, k and v from that of its out; out and lse as it left them (rlkv_packed_attention_grad).

    workspace: a uint8 tensor of rlkv_packed_attention_grad_workspace(tokens, q heads, kv heads) bytes that the caller keeps; without one the
    call takes one from torch's allocator."""
    if workspace is None:
        tokens, q_heads, kv_heads = (*q.shape[:2], k.shape[1]) if q.dim() == 3 and k.dim() == 3 else (0, 1, 1)
        need = load_library().rlkv_packed_attention_grad_workspace(tokens, q_heads, kv_heads)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
    status = _calls.packed_attention_grad(q, k, v, offsets, out, lse, grad_out, grad_q, grad_k, grad_v, scale, _mask_bytes(mask), sink, recent, workspace)
    if status:
        _check(status, "rlkv_packed_attention_grad")
    return grad_q, grad_k, grad_v


def head_norm_rotary(qkv, positions, rotary, q_out, k_out, *, v_out=None, q_weight=None, k_weight=None, eps=None):
    """Norm of every query and key head of packed projections qkv [tokens, (q heads + 2 kv heads) * 128] and rotation by `positions` (int32
    [tokens]) into q_out [tokens, q heads, 128] and k_out [tokens, kv heads, 128] at any strides, values into v_out (rlkv_head_norm_rotary).

    rotary: a Rotary, or None (with positions None): no rotation.  eps None: no norm; weights None: ones.  float32 or bfloat16."""
    status = _calls.head_norm_rotary(qkv, positions, None if rotary is None else rotary.address, q_out, k_out, v_out, q_weight, k_weight, eps)
    if status:
        _check(status, "rlkv_head_norm_rotary")
    return q_out, k_out


def head_norm_rotary_grad(qkv, positions, rotary, grad_q, grad_k, grad_qkv, *, grad_v=None, q_weight=None, k_weight=None, eps=None,
                          grad_q_weight=None, grad_k_weight=None, workspace=None):
    """Gradients of head_norm_rotary's qkv into grad_qkv and of its weights into grad_q_weight and grad_k_weight (float32 [128], where given)
    from those of its outputs; without grad_v the values' columns are left as they are (rlkv_head_norm_rotary_grad).

    workspace: a uint8 tensor of rlkv_head_norm_rotary_grad_workspace(tokens, q heads, kv heads) bytes that the caller keeps; without one the
    call takes one from torch's allocator."""
    if workspace is None:
        tokens, q_heads, kv_heads = (*grad_q.shape[:2], grad_k.shape[1]) if grad_q.dim() == 3 and grad_k.dim() == 3 else (0, 1, 1)
        need = load_library().rlkv_head_norm_rotary_grad_workspace(tokens, q_heads, kv_heads)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=qkv.device)
    status = _calls.head_norm_rotary_grad(qkv, positions, None if rotary is None else rotary.address, grad_q, grad_k, grad_qkv, grad_v,
                                          q_weight, k_weight, eps, grad_q_weight, grad_k_weight, workspace)
    if status:
        _check(status, "rlkv_head_norm_rotary_grad")
    return grad_qkv


def sample_tokens(logits, uniforms, tokens, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logprobs=None, workspace=None):
    """A token of every row of logits [rows, vocab] (float32 or bfloat16) into tokens (int32 [rows]), drawn by uniforms (float32 [rows], in
    [0, 1)) from softmax(logits / temperature) over what top_k, then top_p, then min_p keep, and where given its log probability there into
    logprobs (float32 [rows]) (rlkv_sample_tokens).

    temperature (0: the most likely token), top_k (0: off), top_p (1: off), min_p (0: off): each a number, or a tensor of one a row on the device
    (float32; top_k int32).  workspace: a uint8 tensor of rlkv_sample_tokens_workspace(rows, vocab) bytes that the caller keeps; without one the call
    takes one from torch's allocator."""
    if workspace is None:
        rows, vocab = logits.shape if logits.dim() == 2 else (0, 0)
        need = load_library().rlkv_sample_tokens_workspace(rows, vocab)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=logits.device)
    status = _calls.sample_tokens(logits, uniforms, tokens, temperature, top_k, top_p, min_p, logprobs, workspace)
    if status:
        _check(status, "rlkv_sample_tokens")
    return tokens
