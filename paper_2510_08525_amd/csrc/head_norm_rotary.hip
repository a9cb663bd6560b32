// Queries and keys on their way from the packed projections to an attention without a cache: norm of every head, rotation by the token's
// position; and the way back.  x: a head's 128 values, w: weight, R: rotation (rotary_rows.h),
//
//   y = R(u w),  u = x / sqrt(mean x^2 + eps)            g = R^-1(grad_y),  grad_w = sum g u,  grad_x = (g w - u mean(g w u)) / sqrt(mean x^2 + eps)
//
// Eight threads have a row, 16 values each that stay in registers from the load to the store, so a row is read once and its mean square takes
// three steps over lanes; they keep their token's sines and cosines, and the weight, over several heads.  The weights' gradients are summed
// in registers over all rows that a thread meets, then over the workgroup, whose sums the second launch adds up in a fixed order.
//
// Memory is the bound: 16384 tokens in bf16 of 28 / 4 heads 57 us, 4.7 TB/s, the way back of 32 / 8 heads 110 us, 4.6 TB/s (a large copy reaches 5.1); in
// fp32 121 us, 4.4 TB/s, and 239 us, 4.2 TB/s.
// The next head's rows are asked for before the ones in hand are worked on.  One token: 4.7 us, which is the call's host time.
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

// Queries, keys and values of a token are dealt out in parts, heads of one kind that a thread takes one after the other.
enum Kind { kQuery, kKey, kValue };
struct Deal {
  int32_t heads[3];              // of a token (0 of values: they stay where they are)
  int32_t each[3], parts[3];     // heads of a part, at most; parts of a token
};
Deal deal_of(int tokens, int n_q_heads, int n_kv_heads, bool values) {
  Deal d;
  d.heads[kQuery] = n_q_heads;
  d.heads[kKey] = n_kv_heads;
  d.heads[kValue] = values ? n_kv_heads : 0;
  // (one head each where there are few rows)
  const bool many = (int64_t)tokens * (n_q_heads + n_kv_heads) >= 65536;
  for (int k = 0; k < 3; ++k) {
    d.parts[k] = many ? (d.heads[k] + 7) / 8 : d.heads[k];
    d.each[k] = d.parts[k] ? (d.heads[k] + d.parts[k] - 1) / d.parts[k] : 0;
  }
  return d;
}

// Two pieces of a row as they come from memory.
template <typename T> struct TwoPieces { Piece<T> a, b; };
template <bool STREAM, typename T>
__device__ __forceinline__ TwoPieces<T> two_at(const T* row, int c0, int c1) {
  return {piece_at<STREAM>(row + c0), piece_at<STREAM>(row + c1)};
}
template <typename T>
__device__ __forceinline__ void load_weight(const void* w, int c0, int c1, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = w ? one_value(static_cast<const T*>(w)[c0 + i]) : 1.f;
    f[8 + i] = w ? one_value(static_cast<const T*>(w)[c1 + i]) : 1.f;
  }
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kBlock) void head_norm_rotary_kernel(HeadNormCall c, RotaryTurns turns, Deal deal) {
  const int j = threadIdx.x % kRowThreads, Hq = c.n_q_heads, H = c.n_kv_heads;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const uint32_t parts = deal.parts[0] + deal.parts[1] + deal.parts[2];
  const uint32_t index = blockIdx.x * kItems + threadIdx.x / kRowThreads, token = index / parts;
  int part = (int)(index - token * parts);
  if (token >= (uint32_t)c.tokens) return;
  const int kind = part < deal.parts[0] ? kQuery : part < deal.parts[0] + deal.parts[1] ? kKey : kValue;
  part -= kind == kQuery ? 0 : kind == kKey ? deal.parts[0] : deal.parts[0] + deal.parts[1];
  const int each = kind == kQuery ? deal.each[0] : kind == kKey ? deal.each[1] : deal.each[2], heads = kind == kQuery ? Hq : H;
  const int first = part * each, last = min(first + each, heads);
  const T* row = static_cast<const T*>(c.qkv) + token * c.token_stride + (int64_t)(kind == kQuery ? 0 : kind == kKey ? Hq : Hq + H) * kHeadDim;
  const TokenHeads to = kind == kQuery ? c.q : kind == kKey ? c.k : c.v;
  T* out = static_cast<T*>(to.p) + token * to.token;
  if (first >= last) return;
  TwoPieces<T> next = two_at<STREAM>(row + (int64_t)first * kHeadDim, c0, c1);
  const bool turned = kind != kValue && j < turns.pairs / 8, normed = kind != kValue && c.norm;
  float w[16];
  if (normed) load_weight<T>(kind == kQuery ? c.q_weight : c.k_weight, c0, c1, w);
  Angles g = {};
  if (turned) angles_at(turns, j, c.positions[token], 1.f, g);
  for (int h = first; h < last; ++h) {
    float x[8], y[8];
    widen(next.a, x);
    widen(next.b, y);
    if (h + 1 < last) next = two_at<STREAM>(row + (int64_t)(h + 1) * kHeadDim, c0, c1);
    if (normed) {
      float squares = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += x[i] * x[i] + y[i] * y[i];
      const float r = 1.f / sqrtf(sum_of_row(squares) * (1.f / kHeadDim) + c.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= r * w[i];
        y[i] *= r * w[8 + i];
      }
    }
    if (turned) rotate(turns, g, x, y);
    store_piece<STREAM>(out + h * to.head, c0, kHeadDim, x);
    store_piece<STREAM>(out + h * to.head, c1, kHeadDim, y);
  }
}

// Workgroups [first[k], first[k + 1]) take the parts of kind k, one after the other.
struct GradGrid { int32_t first[4]; };

template <typename T, bool NORM, bool STREAM>
__global__ __launch_bounds__(kBlock) void head_norm_rotary_grad_kernel(HeadNormCall c, RotaryTurns turns, Deal deal, GradGrid grid) {
  const int j = threadIdx.x % kRowThreads, Hq = c.n_q_heads, H = c.n_kv_heads;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const int kind = (int)blockIdx.x < grid.first[1] ? kQuery : (int)blockIdx.x < grid.first[2] ? kKey : kValue;
  const int first_block = kind == kQuery ? 0 : kind == kKey ? grid.first[1] : grid.first[2];
  const int blocks = (kind == kQuery ? grid.first[1] : kind == kKey ? grid.first[2] : grid.first[3]) - first_block;
  const uint32_t parts = kind == kQuery ? deal.parts[0] : kind == kKey ? deal.parts[1] : deal.parts[2];
  const int each = kind == kQuery ? deal.each[0] : kind == kKey ? deal.each[1] : deal.each[2], heads = kind == kQuery ? Hq : H;
  const int64_t column = (int64_t)(kind == kQuery ? 0 : kind == kKey ? Hq : Hq + H) * kHeadDim;
  const TokenHeads from = kind == kQuery ? c.q : kind == kKey ? c.k : c.v;
  const bool turned = kind != kValue && j < turns.pairs / 8, normed = NORM && kind != kValue;
  float w[16], sum[16];
  if (normed) load_weight<T>(kind == kQuery ? c.q_weight : c.k_weight, c0, c1, w);
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  const uint32_t items = (uint32_t)c.tokens * parts;
  for (uint32_t index = (blockIdx.x - first_block) * kItems + threadIdx.x / kRowThreads; index < items; index += blocks * kItems) {
    const uint32_t token = index / parts;
    const int first = (int)(index - token * parts) * each, last = min(first + each, heads);
    const T* row = static_cast<const T*>(c.qkv) + token * c.token_stride + column;
    const T* grad = static_cast<const T*>(from.p) + token * from.token;
    T* out = static_cast<T*>(c.grad) + token * c.grad_stride + column;
    if (first >= last) continue;
    TwoPieces<T> next_g = two_at<STREAM>(grad + first * from.head, c0, c1), next_x = next_g;
    if (normed) next_x = two_at<STREAM>(row + (int64_t)first * kHeadDim, c0, c1);
    Angles g = {};
    if (turned) angles_at(turns, j, c.positions[token], -1.f, g);
    for (int h = first; h < last; ++h) {
      float x[8], y[8], a[8], b[8];
      widen(next_g.a, x);
      widen(next_g.b, y);
      if (normed) {
        widen(next_x.a, a);
        widen(next_x.b, b);
      }
      if (h + 1 < last) {
        next_g = two_at<STREAM>(grad + (h + 1) * from.head, c0, c1);
        if (normed) next_x = two_at<STREAM>(row + (int64_t)(h + 1) * kHeadDim, c0, c1);
      }
      if (turned) rotate(turns, g, x, y);
      if (normed) {
        float squares = 0.f, along = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) squares += a[i] * a[i] + b[i] * b[i];
        const float r = 1.f / sqrtf(sum_of_row(squares) * (1.f / kHeadDim) + c.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] *= r;
          b[i] *= r;
          sum[i] = __builtin_fmaf(x[i], a[i], sum[i]);
          sum[8 + i] = __builtin_fmaf(y[i], b[i], sum[8 + i]);
          x[i] *= w[i];
          y[i] *= w[8 + i];
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
  if (!NORM || !c.partials || kind == kValue) return;
  // over the rows side by side: first within the wavefront (lanes 8 apart), then over the wavefronts
  __shared__ float sums[kBlock / 64][kHeadDim];
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float s = sum[i];
    for (int d = 8; d < 64; d *= 2) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) < kRowThreads) sums[wave][i < 8 ? c0 + i : c1 + i - 8] = s;
  }
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  float total = 0.f;
#pragma unroll
  for (int v = 0; v < kBlock / 64; ++v) total += sums[v][threadIdx.x];
  c.partials[(int64_t)blockIdx.x * kHeadDim + threadIdx.x] = total;
}

// The workgroups' sums of 16 columns of one weight, 64 rows side by side, in 64 bits.
constexpr int kSumThreads = 1024, kSumColumns = 16, kSumRows = kSumThreads / kSumColumns;
__global__ __launch_bounds__(kSumThreads) void weight_grad_kernel(const float* __restrict__ partials, GradGrid grid, float* __restrict__ grad_q,
                                                                  float* __restrict__ grad_k) {
  __shared__ double sums[kSumRows][kSumColumns];
  const int kind = blockIdx.y, col = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns, part = threadIdx.x / kSumColumns;
  float* out = kind == kQuery ? grad_q : grad_k;
  if (!out) return;
  const int first = kind == kQuery ? 0 : grid.first[1], last = kind == kQuery ? grid.first[1] : grid.first[2];
  double sum = 0.;
#pragma unroll 4
  for (int b = first + part; b < last; b += kSumRows) sum += partials[(int64_t)b * kHeadDim + col];
  sums[part][threadIdx.x % kSumColumns] = sum;
  __syncthreads();
  for (int n = kSumRows / 2; n; n /= 2) {
    if (part < n) sums[part][threadIdx.x % kSumColumns] += sums[part + n][threadIdx.x % kSumColumns];
    __syncthreads();
  }
  if (part == 0) out[col] = (float)sums[0][threadIdx.x];
}

constexpr int kGradBlocks = 1024;          // four a compute unit
constexpr int kRowsInTurn = 512;           // rows that a thread adds up one behind the other in fp32, at most: beyond them there are more workgroups

// Workgroups of a kind of head: as many as all its items, as its share of kGradBlocks, and as its weight's sums need at least.
int64_t all_blocks(int64_t tokens, const Deal& d, int k) { return (tokens * d.parts[k] + kItems - 1) / kItems; }
int64_t share_blocks(const Deal& d, int k) {
  const int64_t heads = d.heads[0] + d.heads[1] + d.heads[2];
  return (kGradBlocks * (int64_t)d.heads[k] + heads - 1) / heads;
}
int64_t least_blocks(int64_t tokens, const Deal& d, int k) {
  const int64_t turns = kRowsInTurn / (d.each[k] ? d.each[k] : 1);
  return k == kValue ? 0 : (all_blocks(tokens, d, k) + turns - 1) / turns;
}

template <typename T>
hipError_t launch_forward(const HeadNormCall& c, const RotaryTurns& turns, hipStream_t stream) {
  const Deal deal = deal_of(c.tokens, c.n_q_heads, c.n_kv_heads, c.v.p != nullptr);
  const int64_t items = (int64_t)c.tokens * (deal.parts[0] + deal.parts[1] + deal.parts[2]);
  const int64_t heads = deal.heads[0] + deal.heads[1] + deal.heads[2];
  const bool streams = c.tokens * heads * kHeadDim * 2 * (int64_t)sizeof(T) > kStreamBytes;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((items + kItems - 1) / kItems)), dim3(kBlock), 0, stream, c, turns, deal);
    return hipGetLastError();
  };
  return streams ? launch(head_norm_rotary_kernel<T, true>) : launch(head_norm_rotary_kernel<T, false>);
}
template <typename T>
hipError_t launch_backward(HeadNormCall c, const RotaryTurns& turns, hipStream_t stream) {
  const Deal deal = deal_of(c.tokens, c.n_q_heads, c.n_kv_heads, c.v.p != nullptr);
  const bool sums = c.grad_q_weight || c.grad_k_weight;
  if (!sums) c.partials = nullptr;
  const int64_t heads = deal.heads[0] + deal.heads[1] + deal.heads[2];
  GradGrid grid = {};
  for (int k = 0; k < 3; ++k) {
    const int64_t all = all_blocks(c.tokens, deal, k), share = share_blocks(deal, k), least = least_blocks(c.tokens, deal, k);
    const int64_t blocks = share > least ? share : least;
    grid.first[k + 1] = grid.first[k] + (int)(all < blocks ? all : blocks);
  }
  const bool streams = c.tokens * heads * kHeadDim * 3 * (int64_t)sizeof(T) > kStreamBytes;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid.first[3]), dim3(kBlock), 0, stream, c, turns, deal, grid);
    return hipGetLastError();
  };
  if (c.tokens > 0) {
    const hipError_t err = c.norm ? streams ? launch(head_norm_rotary_grad_kernel<T, true, true>) : launch(head_norm_rotary_grad_kernel<T, true, false>)
                                  : streams ? launch(head_norm_rotary_grad_kernel<T, false, true>) : launch(head_norm_rotary_grad_kernel<T, false, false>);
    if (err != hipSuccess) return err;
  }
  if (!sums) return hipSuccess;
  weight_grad_kernel<<<dim3(kHeadDim / kSumColumns, 2), kSumThreads, 0, stream>>>(c.partials, grid, c.grad_q_weight, c.grad_k_weight);
  return hipGetLastError();
}

}  // namespace

// (No less for more tokens.  A share is rounded up for each kind, and is no smaller where the values have none.)
size_t head_norm_grad_workspace(int tokens, int n_q_heads, int n_kv_heads) {
  const int64_t all = ((int64_t)tokens * (n_q_heads + 2 * (int64_t)n_kv_heads) + kItems - 1) / kItems + 2;
  const Deal deal = deal_of(tokens, n_q_heads, n_kv_heads, true);
  int64_t blocks = kGradBlocks + 3;
  for (int k = kQuery; k <= kKey; ++k) {
    const int64_t share = share_blocks(deal, k), least = least_blocks(tokens, deal, k);
    if (least > share) blocks += least - share;
  }
  return (size_t)(all < blocks ? all : blocks) * kHeadDim * sizeof(float);
}

hipError_t launch_head_norm_rotary(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream) {
  return dtype == RLKV_F32 ? launch_forward<float>(call, turns, stream) : launch_forward<uint16_t>(call, turns, stream);
}
hipError_t launch_head_norm_rotary_grad(const HeadNormCall& call, const RotaryTurns& turns, int dtype, hipStream_t stream) {
  return dtype == RLKV_F32 ? launch_backward<float>(call, turns, stream) : launch_backward<uint16_t>(call, turns, stream);
}

}  // namespace rlkv
