// Norm of every query and key head and rotation by given positions, and the way back: what the host hands to the kernels.
#pragma once

#include "rotary.h"

namespace rlkv {

// Rows of a tensor [tokens][heads][kHeadDim]: element strides.
struct TokenHeads {
  void* p;
  int64_t token, head;
};
struct HeadNormCall {
  const void* qkv;                 // packed projections, rows token_stride elements apart
  int64_t token_stride;
  const int32_t* positions;        // null with turns.pairs == 0
  const void *q_weight, *k_weight; // null: ones
  float eps;
  int32_t norm;                    // 0: rotation alone
  int32_t tokens, n_q_heads, n_kv_heads;
  TokenHeads q, k, v;              // v.p may be null.  Forward: outputs; backward: the gradients of those
  void* grad;                      // backward: packed, rows grad_stride elements apart
  int64_t grad_stride;
  float *grad_q_weight, *grad_k_weight;      // backward, fp32 [kHeadDim]; null: not wanted
  float* partials;                 // backward: [blocks][kHeadDim]
};
hipError_t launch_head_norm_rotary(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream);
hipError_t launch_head_norm_rotary_grad(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream);
size_t head_norm_grad_workspace(int tokens, int n_q_heads, int n_kv_heads);

}  // namespace rlkv
