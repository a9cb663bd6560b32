// What the token-wise operators (norm, quantising, 8-bit product, log probabilities) share: pieces of eight columns, conversions,
// reductions over lanes, and the launchers.
#pragma once

#include "rlkv_internal.h"

namespace rlkv {

constexpr int kGroup = 128;               // columns that share a scale of an 8-bit matrix
constexpr float kE4m3Max = 448.f;         // largest finite value of the 8-bit type (4 exponent, 3 mantissa bits, no infinities)
// The least scale, the smallest normal fp32 number: a group of zeros gets it (and stays zeros), and its reciprocal is finite.
constexpr float kLeastScale = 1.17549435e-38f;

typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef float floats2 __attribute__((ext_vector_type(2)));
typedef float floats4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16s2 __attribute__((ext_vector_type(2)));

// Eight values of a storage type as they come from memory.  They are aligned to one of them only: the hardware takes vector accesses at any
// address, so rows of odd lengths and views that begin anywhere go the same way as others (a gradient of 2048 x 128011 bf16 logits
// into rows without a gap between them: 453 us with their values stored one by one).
template <typename T> struct Piece;
template <> struct Piece<uint16_t> { words4 w; } __attribute__((packed, aligned(2)));
template <> struct Piece<float> { floats4 a, b; } __attribute__((packed, aligned(4)));
typedef words2 words2_at_any_byte __attribute__((aligned(1)));
typedef words2 words2_of_halves __attribute__((aligned(2)));
typedef floats4 floats4_of_floats __attribute__((aligned(4)));

__device__ __forceinline__ void widen(const Piece<uint16_t>& p, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(p.w[i] << 16);
    f[2 * i + 1] = __uint_as_float(p.w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Piece<float>& p, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[i] = p.a[i]; f[4 + i] = p.b[i]; }
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {      // two values rounded to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floats2{a, b}), bf16s2));
}
__device__ __forceinline__ void narrow(const float (&f)[8], Piece<uint16_t>& p) {
#pragma unroll
  for (int i = 0; i < 4; ++i) p.w[i] = bf16_pair(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ void narrow(const float (&f)[8], Piece<float>& p) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { p.a[i] = f[i]; p.b[i] = f[4 + i]; }
}
__device__ __forceinline__ float one_value(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ float one_value(float v) { return v; }
__device__ __forceinline__ void put_value(uint16_t* p, float v) { *p = (uint16_t)bf16_pair(v, 0.f); }
__device__ __forceinline__ void put_value(float* p, float v) { *p = v; }

// STREAM: non-temporal accesses, for what would be gone from the caches before anything asks for it again.
typedef words4 words4_of_halves __attribute__((aligned(2)));
template <bool STREAM>
__device__ __forceinline__ Piece<uint16_t> piece_at(const uint16_t* p) {
  if constexpr (STREAM) return Piece<uint16_t>{__builtin_nontemporal_load(reinterpret_cast<const words4_of_halves*>(p))};
  else return *reinterpret_cast<const Piece<uint16_t>*>(p);
}
template <bool STREAM>
__device__ __forceinline__ Piece<float> piece_at(const float* p) {
  if constexpr (STREAM) {
    const floats4_of_floats* q = reinterpret_cast<const floats4_of_floats*>(p);
    return Piece<float>{__builtin_nontemporal_load(q), __builtin_nontemporal_load(q + 1)};
  } else {
    return *reinterpret_cast<const Piece<float>*>(p);
  }
}
template <bool STREAM>
__device__ __forceinline__ void put_piece(uint16_t* p, const Piece<uint16_t>& v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v.w, reinterpret_cast<words4_of_halves*>(p));
  else *reinterpret_cast<Piece<uint16_t>*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ void put_piece(float* p, const Piece<float>& v) {
  if constexpr (STREAM) {
    floats4_of_floats* q = reinterpret_cast<floats4_of_floats*>(p);
    __builtin_nontemporal_store(v.a, q);
    __builtin_nontemporal_store(v.b, q + 1);
  } else {
    *reinterpret_cast<Piece<float>*>(p) = v;
  }
}
// A call that reads and writes more than the last-level cache holds: what it passes first is gone when it ends.  (Below that, who reads it next
// pays: log probabilities and then gradients of 512 x 128011 bf16 logits 87.0 us with plain loads, 89.7 with non-temporal ones in the first;
// 512 x 32000 22.3 and 25.2; beyond it, 2048 x 128011, 339.6 and 317.4.)
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

// Columns [col, col + 8) of a row of n columns as fp32, zeros past its end.
template <bool STREAM = false, typename T>
__device__ __forceinline__ void load_piece(const T* row, int col, int n, float (&f)[8]) {
  if (col + 8 <= n) {
    widen(piece_at<STREAM>(row + col), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = col + i < n ? one_value(row[col + i]) : 0.f;
  }
}
template <bool STREAM = false, typename T>
__device__ __forceinline__ void store_piece(T* row, int col, int n, const float (&f)[8]) {
  if (col + 8 <= n) {
    Piece<T> p;
    narrow(f, p);
    put_piece<STREAM>(row + col, p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < n) put_value(row + col + i, f[i]);
  }
}
// Eight values as 8-bit ones (rounded to nearest even).
__device__ __forceinline__ void store_e4m3(uint8_t* row, int col, int n, const float (&f)[8]) {
  words2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], lo, true);
  }
  if (col + 8 <= n) {
    *reinterpret_cast<words2_at_any_byte*>(row + col) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < n) row[col + i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

// Over the wavefront, in all lanes (every lane is at the call): within rows of 16 lanes, then over the rows, a vector instruction a step
// where a shuffle is an access to LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_lane(float otherwise, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(otherwise), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float over_wave(float x, float neutral, F f) {
  x = f(x, from_lane<0x111, 0xf>(neutral, x));        // row_shr:1, 2, 4, 8: the row's last lane has the row
  x = f(x, from_lane<0x112, 0xf>(neutral, x));
  x = f(x, from_lane<0x114, 0xf>(neutral, x));
  x = f(x, from_lane<0x118, 0xf>(neutral, x));
  x = f(x, from_lane<0x142, 0xa>(neutral, x));        // row_bcast:15 into rows 1 and 3
  x = f(x, from_lane<0x143, 0xc>(neutral, x));        // row_bcast:31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float sum_of_wave(float x) {
  return over_wave(x, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float max_of_wave(float x) {
  return over_wave(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}

// ---- launchers ---------------------------------------------------------------------------------------------------
// One call of the norm (weight / eps) or of quantising alone (norm false); strides in elements.
struct NormCall {
  const void* x;
  const void* residual;       // or null
  void* sum_out;              // or null (with residual only)
  const void* weight;         // or null: ones
  void* out;
  float* scales;              // [group][row], out_e4m3 only
  int64_t x_stride, residual_stride, sum_stride, out_stride, scale_stride;
  float eps;
  int32_t rows, cols;
  int32_t norm;
};
hipError_t launch_norm(const NormCall& call, int dtype, bool out_e4m3, hipStream_t stream);

// One 8-bit product; strides in elements (bytes for a and b).
struct MatmulCall {
  const void* a;
  const float* a_scales;
  const void* b;
  const float* b_scales;
  void* out;
  int64_t a_stride, a_scale_stride, b_stride, b_scale_stride, out_stride;
  int32_t m, n, k;
};
constexpr int64_t kMostMatmulStride = 1 << 23;         // bytes between rows of a or b: a tile's rows are within 32 bits of its first
hipError_t launch_matmul(const MatmulCall& call, bool out_bf16, hipStream_t stream);
// What a workgroup of the launch has: rows of a, rows of b, parts of k, and the place of that shape among those of its kind, whose number is
// the result (sizes of the call only).
int plan_matmul(const MatmulCall& call, bool out_bf16, int* plan);

constexpr int kMostTop = 32;          // most likely tokens a row can be asked for
struct LogprobCall {
  const void* logits;
  const int32_t* tokens;      // or null (then logprobs is too)
  float* logprobs;
  float* entropy;             // any of these may be null
  float* lse;
  int32_t* top_ids;           // [rows][top], with top > 0
  float* top_logprobs;
  void* workspace;
  int64_t stride;
  float scale;
  int32_t rows, vocab, top;
  int32_t chunks, splits;     // set by the launch
};
struct LogprobGradCall {
  const void* logits;
  const int32_t* tokens;
  const float* lse;
  const float* entropy;
  const float* grad_logprobs;
  const float* grad_entropy;
  void* out;
  int64_t stride, out_stride;
  float scale;
  int32_t rows, vocab;
  int32_t splits;             // set by the launch
};
size_t logprob_workspace(int rows, int vocab, int top);
hipError_t launch_logprobs(LogprobCall call, int dtype, hipStream_t stream);
hipError_t launch_logprobs_grad(LogprobGradCall call, int dtype, hipStream_t stream);

}  // namespace rlkv
