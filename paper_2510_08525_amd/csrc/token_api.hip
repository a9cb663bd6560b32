// Entry points of the token-wise operators: argument checks, all of them before the first HIP call.
#include <math.h>

#include "token_ops.h"

using namespace rlkv;

namespace {

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
size_t bytes_of(int dtype) { return dtype == RLKV_F32 ? 4 : dtype == RLKV_BF16 ? 2 : 1; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int groups_of(int cols) { return (int)(((int64_t)cols + kGroup - 1) / kGroup); }

// A matrix the call reads: rows may repeat (a stride below the columns), but not run backwards.
bool readable(const void* p, int64_t stride, int dtype) { return p && stride >= 0 && aligned(p, bytes_of(dtype)); }
// One that it writes: rows are apart.
bool writable(const void* p, int64_t stride, int64_t rows, int64_t cols, int dtype) {
  return p && (stride >= cols || rows <= 1) && aligned(p, bytes_of(dtype));
}
// Whether every row starts at a multiple of 16 bytes.
bool whole(const void* p, int64_t stride, int dtype) { return aligned(p, 16) && (stride * (int64_t)bytes_of(dtype)) % 16 == 0; }

constexpr int32_t kMostLogitRows = 1 << 20, kMostVocab = 1 << 24;
constexpr float kMostScale = 1.70141183e38f;             // 2^127 (times log2(e) it is still finite)
constexpr int32_t kMostNormCols = 1 << 30;              // (a piece or a stride of threads further on is still an int)

rlkv_status_t norm_call(NormCall& c, int dtype, int out_dtype, void* stream) {
  if (dtype != RLKV_F32 && dtype != RLKV_BF16) return RLKV_ERR_INVALID_ARG;
  if (out_dtype != dtype && out_dtype != RLKV_E4M3) return RLKV_ERR_INVALID_ARG;
  if (c.rows < 0 || c.cols < 1 || c.cols > kMostNormCols) return RLKV_ERR_INVALID_ARG;
  if (c.rows == 0) return RLKV_OK;
  if (!readable(c.x, c.x_stride, dtype) || !writable(c.out, c.out_stride, c.rows, c.cols, out_dtype)) return RLKV_ERR_INVALID_ARG;
  if (c.residual && !readable(c.residual, c.residual_stride, dtype)) return RLKV_ERR_INVALID_ARG;
  if (c.sum_out && (!c.residual || !writable(c.sum_out, c.sum_stride, c.rows, c.cols, dtype))) return RLKV_ERR_INVALID_ARG;
  if (c.weight && !aligned(c.weight, bytes_of(dtype))) return RLKV_ERR_INVALID_ARG;
  const bool e4m3 = out_dtype == RLKV_E4M3;
  if (e4m3 ? !writable(c.scales, c.scale_stride, groups_of(c.cols), c.rows, RLKV_F32) : c.scales != nullptr) return RLKV_ERR_INVALID_ARG;
  return launch_norm(c, dtype, e4m3, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

}  // namespace

extern "C" {

rlkv_status_t rlkv_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                            float eps, int32_t rows, int32_t cols, int32_t dtype, void* sum_out, int64_t sum_stride, void* out,
                            int64_t out_stride, int32_t out_dtype, float* scales, int64_t scale_stride, void* stream) {
  if (!(eps >= 0.f) || isinf(eps)) return RLKV_ERR_INVALID_ARG;
  NormCall c = {};
  c.x = x; c.x_stride = x_stride;
  c.residual = residual; c.residual_stride = residual_stride;
  c.sum_out = sum_out; c.sum_stride = sum_stride;
  c.out = out; c.out_stride = out_stride;
  c.scales = scales; c.scale_stride = scale_stride;
  c.weight = weight; c.eps = eps;
  c.rows = rows; c.cols = cols;
  c.norm = 1;
  return norm_call(c, dtype, out_dtype, stream);
}

rlkv_status_t rlkv_quantize(const void* x, int64_t x_stride, int32_t rows, int32_t cols, int32_t dtype, void* out,
                            int64_t out_stride, float* scales, int64_t scale_stride, void* stream) {
  NormCall c = {};
  c.x = x; c.x_stride = x_stride;
  c.out = out; c.out_stride = out_stride;
  c.scales = scales; c.scale_stride = scale_stride;
  c.rows = rows; c.cols = cols;
  return norm_call(c, dtype, RLKV_E4M3, stream);
}

static bool product_valid(int32_t m, int32_t n, int32_t k, int32_t out_dtype) {
  if (out_dtype != RLKV_F32 && out_dtype != RLKV_BF16) return false;
  if (m < 0 || n < 0 || k < 1 || k % 16 != 0) return false;
  if (m > (1 << 24) || n > (1 << 24) || k > (1 << 24)) return false;
  return (int64_t)(m / 128 + 1) * (n / 128 + 1) <= (1 << 22);      // (threads of a launch are below 2^32)
}

int32_t rlkv_plan_matmul(int32_t m, int32_t n, int32_t k, int32_t out_dtype, int32_t* plan) {
  if (!plan || m < 1 || n < 1 || !product_valid(m, n, k, out_dtype)) return -1;
  MatmulCall c = {};
  c.m = m; c.n = n; c.k = k;
  return plan_matmul(c, out_dtype == RLKV_BF16, plan);
}

rlkv_status_t rlkv_scaled_matmul(const void* a, int64_t a_stride, const float* a_scales, int64_t a_scale_stride, const void* b,
                                 int64_t b_stride, const float* b_scales, int64_t b_scale_stride, int32_t m, int32_t n, int32_t k,
                                 void* out, int64_t out_stride, int32_t out_dtype, void* stream) {
  if (!product_valid(m, n, k, out_dtype)) return RLKV_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return RLKV_OK;
  if (!readable(a, a_stride, RLKV_E4M3) || !readable(b, b_stride, RLKV_E4M3) || !whole(a, a_stride, RLKV_E4M3) ||
      !whole(b, b_stride, RLKV_E4M3) || a_stride > kMostMatmulStride || b_stride > kMostMatmulStride)
    return RLKV_ERR_INVALID_ARG;
  if (!readable(a_scales, a_scale_stride, RLKV_F32) || !readable(b_scales, b_scale_stride, RLKV_F32)) return RLKV_ERR_INVALID_ARG;
  if (!writable(out, out_stride, m, n, out_dtype)) return RLKV_ERR_INVALID_ARG;
  MatmulCall c = {};
  c.a = a; c.a_stride = a_stride;
  c.a_scales = a_scales; c.a_scale_stride = a_scale_stride;
  c.b = b; c.b_stride = b_stride;
  c.b_scales = b_scales; c.b_scale_stride = b_scale_stride;
  c.m = m; c.n = n; c.k = k;
  c.out = out; c.out_stride = out_stride;
  return launch_matmul(c, out_dtype == RLKV_BF16, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

static bool logits_valid(int32_t rows, int32_t vocab, int32_t dtype, float scale) {
  if (dtype != RLKV_F32 && dtype != RLKV_BF16) return false;
  return rows >= 0 && rows <= kMostLogitRows && vocab >= 1 && vocab <= kMostVocab && scale > 0.f && scale <= kMostScale;
}

size_t rlkv_token_logprobs_workspace(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 1 || rows > kMostLogitRows || vocab < 1 || vocab > kMostVocab || top < 0 || top > kMostTop) return 0;
  return logprob_workspace(rows, vocab, top);
}

rlkv_status_t rlkv_token_logprobs(const void* logits, int64_t stride, int32_t rows, int32_t vocab, int32_t dtype, float scale,
                                  const int32_t* tokens, float* logprobs, float* entropy, float* lse, int32_t top, int32_t* top_ids,
                                  float* top_logprobs, void* workspace, size_t workspace_bytes, void* stream) {
  if (!logits_valid(rows, vocab, dtype, scale)) return RLKV_ERR_INVALID_ARG;
  if (top < 0 || top > kMostTop || top > vocab) return RLKV_ERR_INVALID_ARG;
  if (rows == 0) return RLKV_OK;
  if (!readable(logits, stride, dtype)) return RLKV_ERR_INVALID_ARG;
  if ((tokens != nullptr) != (logprobs != nullptr)) return RLKV_ERR_INVALID_ARG;
  if (top > 0 && (!top_ids || !top_logprobs)) return RLKV_ERR_INVALID_ARG;
  if (!aligned(tokens, 4) || !aligned(logprobs, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_ids, 4) ||
      !aligned(top_logprobs, 4) || !aligned(workspace, 8))
    return RLKV_ERR_INVALID_ARG;
  const size_t need = logprob_workspace(rows, vocab, top);
  if (need > 0 && (!workspace || workspace_bytes < need)) return RLKV_ERR_INVALID_ARG;
  LogprobCall c = {};
  c.logits = logits; c.stride = stride;
  c.rows = rows; c.vocab = vocab; c.scale = scale;
  c.tokens = tokens; c.logprobs = logprobs; c.entropy = entropy; c.lse = lse;
  c.top = top; c.top_ids = top_ids; c.top_logprobs = top_logprobs;
  c.workspace = workspace;
  return launch_logprobs(c, dtype, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

rlkv_status_t rlkv_token_logprobs_grad(const void* logits, int64_t stride, int32_t rows, int32_t vocab, int32_t dtype, float scale,
                                       const int32_t* tokens, const float* lse, const float* entropy, const float* grad_logprobs,
                                       const float* grad_entropy, void* grad_logits, int64_t grad_stride, void* stream) {
  if (!logits_valid(rows, vocab, dtype, scale)) return RLKV_ERR_INVALID_ARG;
  if (rows == 0) return RLKV_OK;
  if (!readable(logits, stride, dtype) || !writable(grad_logits, grad_stride, rows, vocab, dtype) || !lse) return RLKV_ERR_INVALID_ARG;
  if ((tokens != nullptr) != (grad_logprobs != nullptr) || (entropy != nullptr) != (grad_entropy != nullptr)) return RLKV_ERR_INVALID_ARG;
  if (!aligned(tokens, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(grad_logprobs, 4) || !aligned(grad_entropy, 4))
    return RLKV_ERR_INVALID_ARG;
  LogprobGradCall c = {};
  c.logits = logits; c.stride = stride;
  c.rows = rows; c.vocab = vocab; c.scale = scale;
  c.tokens = tokens; c.lse = lse; c.entropy = entropy; c.grad_logprobs = grad_logprobs; c.grad_entropy = grad_entropy;
  c.out = grad_logits; c.out_stride = grad_stride;
  return launch_logprobs_grad(c, dtype, as_stream(stream)) == hipSuccess ? RLKV_OK : RLKV_ERR_HIP;
}

}  // extern "C"
