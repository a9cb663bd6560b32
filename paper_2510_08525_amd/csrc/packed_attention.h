// Attention over sequences packed one behind the other: what its kernels (forward and the two of the gradient) share.
//
// Rows of queries, of keys, ... are 128 bf16 values.  The query heads of a KV head are flattened with the positions into columns, position
// first: column c of KV head h is position c / group of query head h * group + c % group.  So a workgroup of few positions still fills its
// matrix instructions, its columns are close to each other in the sequence (the causal diagonal and the edge of the local band cost little),
// and all of them read the same keys.
//
// All products are v_mfma_f32_32x32x16_bf16.  Of its operands lane l holds row (column) l % 32 and the k's 8 (l / 32) .. + 7; of the
// result the column l % 32 and the rows 8 (r / 4) + 4 (l / 32) + r % 4, r = 0 .. 15.  The result of one product is the operand of the
// next without moving: registers 8 s .. 8 s + 7 are the k's {4 half .. + 3, 8 + 4 half .. + 3} of the s-th 16, an order of k that the other operand
// has to have too (transposed_fragment).  So softmax weights never pass through LDS, and what belongs to a column stays in its two lanes.
#pragma once

#include "rlkv_internal.h"

namespace rlkv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef short shorts4 __attribute__((ext_vector_type(4)));

constexpr int kPackedMaskWords = 4;                   // 64 KV heads each
constexpr int kPackedHeads = 64 * kPackedMaskWords;   // KV heads a call can have

// Rows of a tensor [tokens][heads][128]: element strides.
struct HeadRows {
  uint16_t* p;
  int64_t token, head;
};
struct PackedPlan { int32_t items, pad[3]; };      // of the gradient's second launch (packed_attention_grad.hip)
struct PackedCall {
  HeadRows q, k, v, out, grad_out, grad_q, grad_k, grad_v;
  float* lse;                       // [n_q_heads][tokens]
  float* delta;                     // the same (gradient only); set by the launch
  PackedPlan* plan;         // gradient only; set by the launch
  float* slots;                     // the same
  void* workspace;                  // gradient only
  const int32_t* offsets;           // [n_seqs + 1]
  int32_t n_seqs, tokens, n_q_heads, n_kv_heads, group;
  int32_t sink, recent;
  float scale;
  uint64_t full[kPackedMaskWords];  // a bit for each KV head
};
hipError_t launch_packed_attention(const PackedCall& call, hipStream_t stream);
size_t packed_grad_workspace(int tokens, int n_q_heads, int n_kv_heads);
hipError_t launch_packed_attention_grad(PackedCall call, hipStream_t stream);

#ifdef __HIP_DEVICE_COMPILE__
#define RLKV_LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(p))
#endif

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// Which sequence a position belongs to.  Offsets come from device memory, where the host cannot check them: whatever they hold, 0 <= begin <=
// position < end <= tokens.  A position of no sequence has begin = -1.
struct Span { int32_t begin, end; };
constexpr int kOffsetsInLds = 1024;
__device__ __forceinline__ Span span_of(const int32_t* offsets, int n_seqs, int tokens, int position) {
  int lo = 0, hi = n_seqs + 1;                 // the first offset behind the position is in [lo, hi]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] > position) hi = mid;
    else lo = mid + 1;
  }
  if (lo == 0 || lo > n_seqs || position >= tokens) return {-1, -1};
  const int b = offsets[lo - 1], e = offsets[lo];
  return {b < 0 ? 0 : b > position ? position : b, e > tokens ? tokens : e};
}

__device__ __forceinline__ float other_half(float x) {      // the value of the lane 32 away
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}
__device__ __forceinline__ float max_of_halves(float x) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Over the lanes of a wavefront (an int each), to all of them.
__device__ __forceinline__ int min_of_lanes(int x) {
  for (int d = 32; d; d >>= 1) x = min(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int max_of_lanes(int x) {
  for (int d = 32; d; d >>= 1) x = max(x, __shfl_xor(x, d));
  return x;
}

__device__ __forceinline__ uint32_t two_bf16(float a, float b) {      // rounded to nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Rows in LDS: 256 bytes each in 16 units of 16 bytes, of which row r holds unit u at u ^ 2 (r % 8).  Then the 8 rows of which 8 lanes read the
// same unit at a time, and the 4 rows of which 16 lanes read two units transposed, lie in banks of their own.
__device__ __forceinline__ int unit_at(int row, int unit) { return row * 16 + (unit ^ ((row & 7) << 1)); }

// Operand of 32 rows for the k's 16 step .. + 15 as they stand (A: rows of a tile in LDS).
__device__ __forceinline__ bf16x8 row_fragment(const uint4* tile, int row0, int step) {
  const int lane = threadIdx.x & 63;
  return __builtin_bit_cast(bf16x8, tile[unit_at(row0 + (lane & 31), 2 * step + (lane >> 5))]);
}
// Operand of the 32 columns 32 block .. of a tile for 16 of its rows, in the order of k that a product's result has.
__device__ __forceinline__ bf16x8 transposed_fragment(const uint4* tile, int row0, int block) {
#ifdef __HIP_DEVICE_COMPILE__
  const int lane = threadIdx.x & 63;
  const int row = row0 + 4 * (lane >> 5) + ((lane >> 2) & 3);
  const int unit = 4 * block + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
  // (row and row + 8 have the same swizzle)
  const char* at = reinterpret_cast<const char*>(tile + unit_at(row, unit)) + 8 * (lane & 1);
  union { shorts4 part[2]; bf16x8 all; } f;
  f.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLKV_LDS_PTR(shorts4, at));
  f.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLKV_LDS_PTR(shorts4, at + 8 * 256));
  return f.all;
#else
  return bf16x8{};
#endif
}

// 64 rows from `token` on of a head's rows, straight from memory to a tile in LDS; of a workgroup of eight wavefronts, all of them at the call.  Rows from
// `tokens` on are the last one.  (Buffer loads, whose base is the same in all lanes; a row's place from it fits 32 bits.)
constexpr int kStageRows = 64;
constexpr int64_t kMostTokenStride = 1 << 24;
__device__ __forceinline__ void stage_rows(const HeadRows& t, int token, int head, int tokens, uint4* tile) {
#ifdef __HIP_DEVICE_COMPILE__
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const __amdgpu_buffer_rsrc_t from =
      __builtin_amdgcn_make_buffer_rsrc(t.p + (int64_t)token * t.token + (int64_t)head * t.head, 0, 0xffffffff, 0x00027000);
  const int most = tokens - 1 - token;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 8 * wave + 4 * i + (lane >> 4), r = row < most ? row : most;
    const uint32_t at = (uint32_t)r * (uint32_t)(t.token * 2) + ((lane & 15) ^ ((row & 7) << 1)) * 16;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, RLKV_LDS_PTR(void, tile + (8 * wave + 4 * i) * 16), 16, (int)at, 0, 0, 0);
  }
#endif
}

// Results of 16 rows as the operand of the next product: rounded to bf16 (half a step of 2^-8 each, independent of each other: less than what the
// rounding of the output leaves).
__device__ __forceinline__ bf16x8 weights_fragment(const floatx16& x, int step) {
  words4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = two_bf16(x[8 * step + 2 * i], x[8 * step + 2 * i + 1]);
  return __builtin_bit_cast(bf16x8, w);
}

}  // namespace rlkv
