// Entry points of the policy's training loop: argument checks, all of them before the first HIP call.
#include <math.h>

#include "head_norm_rotary.h"
#include "packed_attention.h"
#include "sample_tokens.h"

using namespace rlkv;

namespace {

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int32_t kMostLogitRows = 1 << 20, kMostVocab = 1 << 24;
constexpr int64_t kMostStride = (int64_t)1 << 40;          // (a row's address is far from 64 bits)

// Rows that the call reads: they may repeat, but not run backwards.
bool readable(const rlkv_heads_t* t, size_t bytes) {
  const int64_t row = 16 / (int64_t)bytes;
  return t && t->data && aligned(t->data, 16) && t->token_stride >= 0 && t->head_stride >= 0 && t->token_stride <= kMostStride &&
         t->head_stride <= kMostStride && t->token_stride % row == 0 && t->head_stride % row == 0;
}
// Rows that it writes: apart from each other, either heads within a token or tokens within a head.
bool writable(const rlkv_heads_t* t, size_t bytes, int64_t tokens, int64_t heads) {
  if (!readable(t, bytes)) return false;
  const int64_t token = t->token_stride, head = t->head_stride;
  const bool heads_inside = (heads <= 1 || head >= kHeadDim) && (tokens <= 1 || token >= (heads - 1) * head + kHeadDim);
  const bool tokens_inside = (tokens <= 1 || token >= kHeadDim) && (heads <= 1 || head >= (tokens - 1) * token + kHeadDim);
  return heads_inside || tokens_inside;
}
HeadRows rows_of(const rlkv_heads_t* t) { return {static_cast<uint16_t*>(t->data), t->token_stride, t->head_stride}; }

bool heads_valid(int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads) {
  if (tokens < 0 || n_kv_heads < 1 || n_kv_heads > kPackedHeads || n_q_heads < 1 || n_q_heads % n_kv_heads != 0) return false;
  const int group = n_q_heads / n_kv_heads;
  return group <= kMaxGroup && (int64_t)tokens * n_q_heads < ((int64_t)1 << 30);      // (two threads a column, below 2^32)
}
constexpr float kLeastSoftmaxScale = 8.67361738e-19f;          // 2^-60
// Rows of a packed call: a tile's 64 are within 32 bits of its first.
bool packed_rows(const rlkv_heads_t* t) { return readable(t, 2) && t->token_stride <= kMostTokenStride; }
bool packed_out(const rlkv_heads_t* t, int64_t tokens, int64_t heads) { return writable(t, 2, tokens, heads) && t->token_stride <= kMostTokenStride; }
bool packed_valid(const rlkv_packed_t* s) {
  if (!s || !heads_valid(s->tokens, s->n_q_heads, s->n_kv_heads)) return false;
  if (s->n_seqs < 0 || s->n_seqs == INT32_MAX || s->sink < 0) return false;
  if (!(s->softmax_scale >= kLeastSoftmaxScale && s->softmax_scale <= 1.f / kLeastSoftmaxScale)) return false;
  for (int h = 0; s->full_mask && h < s->n_kv_heads; ++h)
    if (s->full_mask[h] > 1 || (s->full_mask[h] == 0 && s->recent < 1)) return false;
  return true;
}
PackedCall packed_call(const rlkv_packed_t* s) {
  PackedCall c = {};
  c.offsets = s->offsets;
  c.n_seqs = s->n_seqs;
  c.tokens = s->tokens;
  c.n_q_heads = s->n_q_heads;
  c.n_kv_heads = s->n_kv_heads;
  c.group = s->n_q_heads / s->n_kv_heads;
  c.sink = s->sink;
  c.recent = s->recent;
  c.scale = s->softmax_scale;
  for (int h = 0; h < s->n_kv_heads; ++h)
    if (!s->full_mask || s->full_mask[h]) {
      c.full[h >> 6] |= (uint64_t)1 << (h & 63);
      ++c.n_full;
    }
  c.by_group = Divisor::by(c.group);
  c.by_full = Divisor::by(c.n_full ? c.n_full : 1);
  c.by_local = Divisor::by(c.n_full < c.n_kv_heads ? c.n_kv_heads - c.n_full : 1);
  return c;
}

TokenHeads token_heads(const rlkv_heads_t* t) { return {t->data, t->token_stride, t->head_stride}; }
constexpr int32_t kMostHeads = 1 << 16;
bool head_norm_valid(int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t dtype) {
  if (dtype != RLKV_F32 && dtype != RLKV_BF16) return false;
  if (tokens < 0 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads > kMostHeads || n_kv_heads > kMostHeads) return false;
  return (int64_t)tokens * (n_q_heads + 2 * (int64_t)n_kv_heads) < ((int64_t)1 << 29);      // (eight threads a row, below 2^32)
}
// What both directions have: false where it is wrong.
bool head_norm_call(HeadNormCall* c, RotaryTurns* turns, const void* qkv, int64_t token_stride, const int32_t* positions,
                    const rlkv_rotary_t* rotary, const rlkv_head_norm_t* norm, int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads,
                    int32_t dtype) {
  if (!head_norm_valid(tokens, n_q_heads, n_kv_heads, dtype)) return false;
  *c = {};
  *turns = {};
  if (rotary && (!turns_of(rotary, turns) || (tokens > 0 && !positions) || !aligned(positions, 4))) return false;
  const size_t e = dtype == RLKV_F32 ? 4 : 2;
  if (norm) {
    if (!(norm->eps >= 0.f) || isinf(norm->eps) || !aligned(norm->q_weight, e) || !aligned(norm->k_weight, e)) return false;
    c->norm = 1;
    c->eps = norm->eps;
    c->q_weight = norm->q_weight;
    c->k_weight = norm->k_weight;
  }
  const int64_t width = (n_q_heads + 2 * (int64_t)n_kv_heads) * kHeadDim;
  if (tokens > 0 && (!qkv || !aligned(qkv, e) || token_stride < width || token_stride > kMostStride)) return false;
  c->qkv = qkv;
  c->token_stride = token_stride;
  c->positions = positions;
  c->tokens = tokens;
  c->n_q_heads = n_q_heads;
  c->n_kv_heads = n_kv_heads;
  return true;
}

}  // namespace

extern "C" {

size_t rlkv_sample_tokens_workspace(int32_t rows, int32_t vocab) {
  return rows < 1 || rows > kMostLogitRows || vocab < 1 || vocab > kMostVocab ? 0 : sample_workspace(rows, vocab);
}

rlkv_status_t rlkv_sample_tokens(const void* logits, int64_t stride, int32_t rows, int32_t vocab, int32_t dtype, const rlkv_sampling_t* how,
                                 const float* uniforms, int32_t* tokens, float* logprobs, void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != RLKV_F32 && dtype != RLKV_BF16) return RLKV_ERR_INVALID_ARG;
  if (rows < 0 || rows > kMostLogitRows || vocab < 1 || vocab > kMostVocab || !how) return RLKV_ERR_INVALID_ARG;
  if ((!how->temperatures && (!(how->temperature >= 0.) || isinf(how->temperature))) || (!how->top_ks && how->top_k < 0) ||
      (!how->top_ps && !(how->top_p >= 0.)) || (!how->min_ps && !(how->min_p >= 0. && how->min_p <= 1.)))
    return RLKV_ERR_INVALID_ARG;
  if (!aligned(how->temperatures, 4) || !aligned(how->top_ks, 4) || !aligned(how->top_ps, 4) || !aligned(how->min_ps, 4)) return RLKV_ERR_INVALID_ARG;
  if (rows == 0) return RLKV_OK;
  if (!logits || !aligned(logits, dtype == RLKV_F32 ? 4 : 2) || stride < 0 || stride > kMostStride) return RLKV_ERR_INVALID_ARG;
  if (!uniforms || !tokens || !aligned(uniforms, 4) || !aligned(tokens, 4) || !aligned(logprobs, 4)) return RLKV_ERR_INVALID_ARG;
  const size_t need = sample_workspace(rows, vocab);
  if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return RLKV_ERR_INVALID_ARG;
  SampleCall c = {};
  c.logits = logits;
  c.stride = stride;
  c.rows = rows;
  c.vocab = vocab;
  c.temperature = how->temperature;
  c.top_k = how->top_k;
  c.top_p = how->top_p;
  c.min_p = how->min_p;
  c.temperatures = how->temperatures;
  c.top_ks = how->top_ks;
  c.top_ps = how->top_ps;
  c.min_ps = how->min_ps;
  c.uniforms = uniforms;
  c.tokens = tokens;
  c.logprobs = logprobs;
  c.workspace = workspace;
  return launch_sample(c, dtype, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

rlkv_status_t rlkv_head_norm_rotary(const void* qkv, int64_t token_stride, const int32_t* positions, const rlkv_rotary_t* rotary,
                                    const rlkv_head_norm_t* norm, int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t dtype,
                                    const rlkv_heads_t* q_out, const rlkv_heads_t* k_out, const rlkv_heads_t* v_out, void* stream) {
  HeadNormCall c;
  RotaryTurns turns;
  if (!head_norm_call(&c, &turns, qkv, token_stride, positions, rotary, norm, tokens, n_q_heads, n_kv_heads, dtype)) return RLKV_ERR_INVALID_ARG;
  if (tokens == 0) return RLKV_OK;
  const size_t e = dtype == RLKV_F32 ? 4 : 2;
  if (!writable(q_out, e, tokens, n_q_heads) || !writable(k_out, e, tokens, n_kv_heads) || (v_out && !writable(v_out, e, tokens, n_kv_heads)))
    return RLKV_ERR_INVALID_ARG;
  c.q = token_heads(q_out);
  c.k = token_heads(k_out);
  if (v_out) c.v = token_heads(v_out);
  return launch_head_norm_rotary(c, turns, dtype, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

size_t rlkv_head_norm_rotary_grad_workspace(int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads) {
  if (tokens < 1 || !head_norm_valid(tokens, n_q_heads, n_kv_heads, RLKV_F32)) return 0;
  return head_norm_grad_workspace(tokens, n_q_heads, n_kv_heads);
}

rlkv_status_t rlkv_head_norm_rotary_grad(const void* qkv, int64_t token_stride, const int32_t* positions, const rlkv_rotary_t* rotary,
                                         const rlkv_head_norm_t* norm, int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t dtype,
                                         const rlkv_heads_t* grad_q, const rlkv_heads_t* grad_k, const rlkv_heads_t* grad_v, void* grad_qkv,
                                         int64_t grad_stride, float* grad_q_weight, float* grad_k_weight, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  HeadNormCall c;
  RotaryTurns turns;
  if (!head_norm_call(&c, &turns, qkv, token_stride, positions, rotary, norm, tokens, n_q_heads, n_kv_heads, dtype)) return RLKV_ERR_INVALID_ARG;
  const bool sums = grad_q_weight || grad_k_weight;
  if (sums && !norm) return RLKV_ERR_INVALID_ARG;
  if (!aligned(grad_q_weight, 4) || !aligned(grad_k_weight, 4)) return RLKV_ERR_INVALID_ARG;
  if (tokens == 0 && !sums) return RLKV_OK;
  if (tokens > 0) {
    const size_t e = dtype == RLKV_F32 ? 4 : 2;
    if (!readable(grad_q, e) || !readable(grad_k, e) || (grad_v && !readable(grad_v, e))) return RLKV_ERR_INVALID_ARG;
    if (!grad_qkv || !aligned(grad_qkv, e) || grad_stride > kMostStride ||
        grad_stride < (n_q_heads + 2 * (int64_t)n_kv_heads) * kHeadDim)
      return RLKV_ERR_INVALID_ARG;
    if (sums && (!workspace || !aligned(workspace, 16) || workspace_bytes < head_norm_grad_workspace(tokens, n_q_heads, n_kv_heads)))
      return RLKV_ERR_INVALID_ARG;
    c.q = token_heads(grad_q);
    c.k = token_heads(grad_k);
    if (grad_v) c.v = token_heads(grad_v);
  }
  c.grad = grad_qkv;
  c.grad_stride = grad_stride;
  c.grad_q_weight = grad_q_weight;
  c.grad_k_weight = grad_k_weight;
  c.partials = static_cast<float*>(workspace);
  return launch_head_norm_rotary_grad(c, turns, dtype, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

rlkv_status_t rlkv_packed_attention(const rlkv_packed_t* shape, const rlkv_heads_t* q, const rlkv_heads_t* k, const rlkv_heads_t* v,
                                    const rlkv_heads_t* out, float* lse, void* stream) {
  if (!packed_valid(shape)) return RLKV_ERR_INVALID_ARG;
  if (shape->tokens == 0 || shape->n_seqs == 0) return RLKV_OK;
  if (!shape->offsets || !aligned(shape->offsets, 4) || !aligned(lse, 4)) return RLKV_ERR_INVALID_ARG;
  if (!packed_rows(q) || !packed_rows(k) || !packed_rows(v)) return RLKV_ERR_INVALID_ARG;
  if (!packed_out(out, shape->tokens, shape->n_q_heads)) return RLKV_ERR_INVALID_ARG;
  PackedCall c = packed_call(shape);
  c.q = rows_of(q);
  c.k = rows_of(k);
  c.v = rows_of(v);
  c.out = rows_of(out);
  c.lse = lse;
  return launch_packed_attention(c, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

size_t rlkv_packed_attention_grad_workspace(int32_t tokens, int32_t n_q_heads, int32_t n_kv_heads) {
  if (tokens < 1 || !heads_valid(tokens, n_q_heads, n_kv_heads)) return 0;
  return packed_grad_workspace(tokens, n_q_heads, n_kv_heads);
}

rlkv_status_t rlkv_packed_attention_grad(const rlkv_packed_t* shape, const rlkv_heads_t* q, const rlkv_heads_t* k, const rlkv_heads_t* v,
                                         const rlkv_heads_t* out, const float* lse, const rlkv_heads_t* grad_out,
                                         const rlkv_heads_t* grad_q, const rlkv_heads_t* grad_k, const rlkv_heads_t* grad_v,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!packed_valid(shape)) return RLKV_ERR_INVALID_ARG;
  if (shape->tokens == 0 || shape->n_seqs == 0) return RLKV_OK;
  if (!shape->offsets || !aligned(shape->offsets, 4) || !lse || !aligned(lse, 4)) return RLKV_ERR_INVALID_ARG;
  if (!packed_rows(q) || !packed_rows(k) || !packed_rows(v) || !packed_rows(out) || !packed_rows(grad_out)) return RLKV_ERR_INVALID_ARG;
  if (!packed_out(grad_q, shape->tokens, shape->n_q_heads) || !packed_out(grad_k, shape->tokens, shape->n_kv_heads) ||
      !packed_out(grad_v, shape->tokens, shape->n_kv_heads))
    return RLKV_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < packed_grad_workspace(shape->tokens, shape->n_q_heads, shape->n_kv_heads))
    return RLKV_ERR_INVALID_ARG;
  PackedCall c = packed_call(shape);
  c.q = rows_of(q);
  c.k = rows_of(k);
  c.v = rows_of(v);
  c.out = rows_of(out);
  c.lse = const_cast<float*>(lse);
  c.grad_out = rows_of(grad_out);
  c.grad_q = rows_of(grad_q);
  c.grad_k = rows_of(grad_k);
  c.grad_v = rows_of(grad_v);
  c.workspace = workspace;
  return launch_packed_attention_grad(c, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

}  // extern "C"
