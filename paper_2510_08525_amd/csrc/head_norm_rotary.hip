// Queries and keys on their way from the packed projections to an attention without a cache: norm of every head, rotation by the token's
// position; and the way back.  x: a head's 128 values, w: weight, R: rotation (rotary_rows.h),
//
//   y = R(u w),  u = x / sqrt(mean x^2 + eps)            g = R^-1(grad_y),  grad_w = sum g u,  grad_x = (g w - u mean(g w u)) / sqrt(mean x^2 + eps)
//
// Eight threads have a row, 16 values each that stay in registers from the load to the store, so a row is read once and its mean square takes
// three steps over lanes; they keep their token's sines and cosines, and the weight, over several heads.  The weights' gradients are summed
// in registers over all rows that a thread meets, then over the workgroup, whose sums the second launch adds up in a fixed order.
#include "head_norm_rotary.h"
#include "rotary_rows.h"
#include "token_ops.h"

namespace rlkv {
namespace {

constexpr int kItems = kBlock / kRowThreads;       // rows a workgroup works on side by side

// Over the eight threads of a row.
__device__ __forceinline__ float sum_of_row(float x) {
  x += from_lane<0xb1, 0xf>(0.f, x);               // quad_perm: lane ^ 1
  x += from_lane<0x4e, 0xf>(0.f, x);               // quad_perm: lane ^ 2
  return x + from_lane<0x141, 0xf>(0.f, x);        // row_half_mirror: the other four
}
__device__ __forceinline__ void angles_at(const RotaryTurns& turns, int j, int position, float direction, Angles& g) {
  angles_of(turns, j, (uint32_t)(position < 0 ? -(int64_t)position : position), g);
  if (position < 0) direction = -direction;
#pragma unroll
  for (int i = 0; i < 8; ++i) g.sine[i] *= direction;
}

// A part of a token's heads: token, first and last head.
struct Part { int64_t token; int first, last; };
__device__ __forceinline__ Part part_of(int64_t index, int parts, int heads_each, int heads) {
  Part p;
  p.token = index / parts;
  p.first = (int)(index - p.token * parts) * heads_each;
  p.last = p.first + heads_each < heads ? p.first + heads_each : heads;
  return p;
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kBlock) void head_norm_rotary_kernel(HeadNormCall c, RotaryTurns turns, int heads, int heads_each) {
  const int j = threadIdx.x % kRowThreads, Hq = c.n_q_heads, H = c.n_kv_heads;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const bool turned = j < turns.pairs / 8;
  const int parts = (heads + heads_each - 1) / heads_each;
  const Part p = part_of((int64_t)blockIdx.x * kItems + threadIdx.x / kRowThreads, parts, heads_each, heads);
  if (p.token >= c.tokens) return;
  const T* row = static_cast<const T*>(c.qkv) + p.token * c.token_stride;
  Angles g = {};
  if (turned && p.first < Hq + H) angles_at(turns, j, c.positions[p.token], 1.f, g);
  float wq[16], wk[16];
  auto weights = [&](const void* w, float (&f)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = w ? one_value(static_cast<const T*>(w)[c0 + i]) : 1.f;
      f[8 + i] = w ? one_value(static_cast<const T*>(w)[c1 + i]) : 1.f;
    }
  };
  if (c.norm && p.first < Hq) weights(c.q_weight, wq);
  if (c.norm && p.last > Hq) weights(c.k_weight, wk);
  for (int h = p.first; h < p.last; ++h) {
    float x[8], y[8];
    load_piece<STREAM>(row + (int64_t)h * kHeadDim, c0, kHeadDim, x);
    load_piece<STREAM>(row + (int64_t)h * kHeadDim, c1, kHeadDim, y);
    if (c.norm && h < Hq + H) {
      float squares = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += x[i] * x[i] + y[i] * y[i];
      const float r = 1.f / sqrtf(sum_of_row(squares) * (1.f / kHeadDim) + c.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= r * (h < Hq ? wq[i] : wk[i]);
        y[i] *= r * (h < Hq ? wq[8 + i] : wk[8 + i]);
      }
    }
    if (turned && h < Hq + H) rotate(turns, g, x, y);
    const TokenHeads& to = h < Hq ? c.q : h < Hq + H ? c.k : c.v;
    T* out = static_cast<T*>(to.p) + p.token * to.token + (h < Hq ? h : h < Hq + H ? h - Hq : h - Hq - H) * to.head;
    store_piece<STREAM>(out, c0, kHeadDim, x);
    store_piece<STREAM>(out, c1, kHeadDim, y);
  }
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kBlock) void head_norm_rotary_grad_kernel(HeadNormCall c, RotaryTurns turns, int heads, int heads_each, int64_t items) {
  const int j = threadIdx.x % kRowThreads, Hq = c.n_q_heads, H = c.n_kv_heads;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const bool turned = j < turns.pairs / 8;
  const int parts = (heads + heads_each - 1) / heads_each;
  float wq[16], wk[16], gq[16], gk[16];
  auto weights = [&](const void* w, float (&f)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = w ? one_value(static_cast<const T*>(w)[c0 + i]) : 1.f;
      f[8 + i] = w ? one_value(static_cast<const T*>(w)[c1 + i]) : 1.f;
    }
  };
  if (c.norm) {
    weights(c.q_weight, wq);
    weights(c.k_weight, wk);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) gq[i] = gk[i] = 0.f;
  for (int64_t index = (int64_t)blockIdx.x * kItems + threadIdx.x / kRowThreads; index < items; index += (int64_t)gridDim.x * kItems) {
    const Part p = part_of(index, parts, heads_each, heads);
    const T* row = static_cast<const T*>(c.qkv) + p.token * c.token_stride;
    T* out = static_cast<T*>(c.grad) + p.token * c.grad_stride;
    Angles g = {};
    if (turned && p.first < Hq + H) angles_at(turns, j, c.positions[p.token], -1.f, g);
    for (int h = p.first; h < p.last; ++h) {
      const TokenHeads& from = h < Hq ? c.q : h < Hq + H ? c.k : c.v;
      const T* grad = static_cast<const T*>(from.p) + p.token * from.token + (h < Hq ? h : h < Hq + H ? h - Hq : h - Hq - H) * from.head;
      float x[8], y[8];
      load_piece<STREAM>(grad, c0, kHeadDim, x);
      load_piece<STREAM>(grad, c1, kHeadDim, y);
      if (turned && h < Hq + H) rotate(turns, g, x, y);
      if (c.norm && h < Hq + H) {
        float a[8], b[8], squares = 0.f, along = 0.f;
        load_piece<STREAM>(row + (int64_t)h * kHeadDim, c0, kHeadDim, a);
        load_piece<STREAM>(row + (int64_t)h * kHeadDim, c1, kHeadDim, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) squares += a[i] * a[i] + b[i] * b[i];
        const float r = 1.f / sqrtf(sum_of_row(squares) * (1.f / kHeadDim) + c.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] *= r;
          b[i] *= r;
          if (h < Hq) {
            gq[i] = __builtin_fmaf(x[i], a[i], gq[i]);
            gq[8 + i] = __builtin_fmaf(y[i], b[i], gq[8 + i]);
          } else {
            gk[i] = __builtin_fmaf(x[i], a[i], gk[i]);
            gk[8 + i] = __builtin_fmaf(y[i], b[i], gk[8 + i]);
          }
          x[i] *= h < Hq ? wq[i] : wk[i];
          y[i] *= h < Hq ? wq[8 + i] : wk[8 + i];
          along = __builtin_fmaf(x[i], a[i], along);
          along = __builtin_fmaf(y[i], b[i], along);
        }
        along = sum_of_row(along) * (1.f / kHeadDim);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = r * __builtin_fmaf(-a[i], along, x[i]);
          y[i] = r * __builtin_fmaf(-b[i], along, y[i]);
        }
      }
      store_piece<STREAM>(out + (int64_t)h * kHeadDim, c0, kHeadDim, x);
      store_piece<STREAM>(out + (int64_t)h * kHeadDim, c1, kHeadDim, y);
    }
  }
  if (!c.partials) return;
  // over the rows side by side: first within the wavefront (lanes 8 apart), then over the wavefronts
  __shared__ float sums[kBlock / 64][2][kHeadDim];
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float q = gq[i], k = gk[i];
    for (int d = 8; d < 64; d *= 2) {
      q += __shfl_xor(q, d);
      k += __shfl_xor(k, d);
    }
    if ((threadIdx.x & 63) < kRowThreads) {
      const int col = i < 8 ? c0 + i : c1 + i - 8;
      sums[wave][0][col] = q;
      sums[wave][1][col] = k;
    }
  }
  __syncthreads();
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kBlock / 64; ++w) total += sums[w][threadIdx.x >> 7][threadIdx.x & 127];
  c.partials[(int64_t)blockIdx.x * 2 * kHeadDim + threadIdx.x] = total;
}
static_assert(kBlock == 2 * kHeadDim, "a thread of the last step has a column of one weight");

// The workgroups' sums of 32 of the 256 columns, eight rows side by side, in 64 bits.
__global__ __launch_bounds__(kBlock) void weight_grad_kernel(const float* __restrict__ partials, int blocks, float* __restrict__ grad_q,
                                                             float* __restrict__ grad_k) {
  __shared__ double sums[8][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
  double sum = 0.;
  for (int b = part; b < blocks; b += 8) sum += partials[(int64_t)b * 2 * kHeadDim + col];
  sums[part][threadIdx.x & 31] = sum;
  __syncthreads();
  if (part != 0) return;
  for (int i = 1; i < 8; ++i) sum += sums[i][threadIdx.x];
  float* out = col < kHeadDim ? grad_q : grad_k;
  if (out) out[col & (kHeadDim - 1)] = (float)sum;
}

// Heads a thread takes one after the other: few where there are few rows.
int heads_each_of(int64_t rows) { return rows >= 65536 ? 8 : 1; }

constexpr int kGradBlocks = 1024;
int64_t grad_items(const HeadNormCall& c, int heads, int heads_each) { return (int64_t)c.tokens * ((heads + heads_each - 1) / heads_each); }

template <typename T>
hipError_t launch_forward(const HeadNormCall& c, const RotaryTurns& turns, hipStream_t stream) {
  const int heads = c.n_q_heads + c.n_kv_heads * (c.v.p ? 2 : 1);
  const int heads_each = heads_each_of((int64_t)c.tokens * heads);
  const int64_t blocks = (grad_items(c, heads, heads_each) + kItems - 1) / kItems;
  const bool streams = (int64_t)c.tokens * heads * kHeadDim * 2 * (int64_t)sizeof(T) > kStreamBytes;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, c, turns, heads, heads_each);
    return hipGetLastError();
  };
  return streams ? launch(head_norm_rotary_kernel<T, true>) : launch(head_norm_rotary_kernel<T, false>);
}
template <typename T>
hipError_t launch_backward(HeadNormCall c, const RotaryTurns& turns, hipStream_t stream) {
  const int heads = c.n_q_heads + c.n_kv_heads * (c.v.p ? 2 : 1);
  const int heads_each = heads_each_of((int64_t)c.tokens * heads);
  const int64_t items = grad_items(c, heads, heads_each), all = (items + kItems - 1) / kItems;
  const bool sums = c.grad_q_weight || c.grad_k_weight;
  if (!sums) c.partials = nullptr;
  const int blocks = (int)(all < kGradBlocks ? all : kGradBlocks);
  const bool streams = (int64_t)c.tokens * heads * kHeadDim * 3 * (int64_t)sizeof(T) > kStreamBytes;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, c, turns, heads, heads_each, items);
    return hipGetLastError();
  };
  if (blocks > 0) {
    const hipError_t err = streams ? launch(head_norm_rotary_grad_kernel<T, true>) : launch(head_norm_rotary_grad_kernel<T, false>);
    if (err != hipSuccess) return err;
  }
  if (!sums) return hipSuccess;
  weight_grad_kernel<<<2 * kHeadDim / 32, kBlock, 0, stream>>>(c.partials, blocks, c.grad_q_weight, c.grad_k_weight);
  return hipGetLastError();
}

}  // namespace

size_t head_norm_grad_workspace(int tokens, int n_q_heads, int n_kv_heads) {
  const int64_t all = ((int64_t)tokens * (n_q_heads + 2 * (int64_t)n_kv_heads) + kItems - 1) / kItems;
  return (size_t)(all < kGradBlocks ? all : kGradBlocks) * 2 * kHeadDim * sizeof(float);
}

hipError_t launch_head_norm_rotary(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream) {
  return dtype == RLKV_F32 ? launch_forward<float>(call, turns, stream) : launch_forward<uint16_t>(call, turns, stream);
}
hipError_t launch_head_norm_rotary_grad(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream) {
  return dtype == RLKV_F32 ? launch_backward<float>(call, turns, stream) : launch_backward<uint16_t>(call, turns, stream);
}

}  // namespace rlkv
