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

#include <type_traits>

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

// Result [d][column] as a row of the column's lanes: 16 bytes of it a store (the halves of the wavefront swap words).
__device__ __forceinline__ void store_rows(uint16_t* row, const floatx16 (&x)[4], float scale, bool valid) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      words4 w;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t even = two_bf16(x[b][4 * g + 2 * i] * scale, x[b][4 * g + 2 * i + 1] * scale);
        const uint32_t odd = two_bf16(x[b][4 * g + 4 + 2 * i] * scale, x[b][4 * g + 5 + 2 * i] * scale);
        const u32x2 r = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
        w[i] = r[0];
        w[2 + i] = r[1];
      }
      if (valid) *reinterpret_cast<words4*>(row + 32 * b + 8 * (g + half)) = w;
    }
}

// x * 0 summed: 0, or NaN where any is not finite.
__device__ __forceinline__ float zero_or_nan(const floatx16 (&x)[4]) {
  float all = 0.f;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) all += x[b][r] * 0.f;
  return all;
}
__device__ __forceinline__ void clear(floatx16& x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 0.f;
}
// acc[d][column] += sum over the rows of a 32-row tile of tile[row][d] * w[row][column] of admitted pairs, without the matrix instruction: a
// weight of 0 does not keep an infinity or a NaN in the tile out of its products.
template <typename F>
__device__ __forceinline__ void admitted_products(const uint4* tile, int row0, const floatx16& w, floatx16 (&acc)[4], F admits) {
  const int half = (threadIdx.x >> 5) & 1;
  for (int row = 0; row < 32; ++row) {
    float x = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r >> 2) + (r & 3) == (row & ~4)) x = w[r];
    const float other = other_half(x);
    if (((row >> 2) & 1) != half) x = other;
    if (!admits(row)) continue;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * b + 8 * g + 4 * half;
        const words2 two = *reinterpret_cast<const words2*>(reinterpret_cast<const char*>(tile + unit_at(row0 + row, d >> 3)) + 2 * (d & 7));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][4 * g + e] += x * __uint_as_float(e & 1 ? two[e >> 1] & 0xffff0000u : two[e >> 1] << 16);
      }
  }
}

// ---- a workgroup of 256 columns and the tiles of keys that it walks over ----
constexpr int kPackedWaves = 8, kPackedThreads = 64 * kPackedWaves;
constexpr int kColumns = 32 * kPackedWaves, kKeys = kStageRows;

// The n-th KV head of a launch: full ones in front of local ones, so that the long workgroups are handed out first, and neighbours in the launch
// (which the hardware deals to the 8 XCDs in turn) are of different heads: a head's keys are then read by few of the L2s.
__device__ __forceinline__ int head_in_order(const PackedCall& c, int n, bool& full) {
  int n_full = 0;
  for (int w = 0; w < kPackedMaskWords; ++w) n_full += __popcll(c.full[w]);
  full = n < n_full;
  if (!full) n -= n_full;
  for (int w = 0;; ++w) {
    uint64_t bits = full ? c.full[w] : ~c.full[w];
    const int here = __popcll(bits);
    if (n >= here) {
      n -= here;
      continue;
    }
    for (; n; --n) bits &= bits - 1;
    return w * 64 + __builtin_ctzll(bits);
  }
}
// Block and head of the launch's workgroup `index`: of all full heads the last blocks first, then of the local ones.
struct ColumnBlock { int block, head; bool full; };
__device__ __forceinline__ ColumnBlock column_block(const PackedCall& c, uint32_t index, uint32_t blocks) {
  int n_full = 0;
  for (int w = 0; w < kPackedMaskWords; ++w) n_full += __popcll(c.full[w]);
  ColumnBlock b;
  uint32_t n;
  if (index < blocks * n_full) {
    b.block = blocks - 1 - index / n_full;
    n = index % n_full;
  } else {
    index -= blocks * n_full;
    const uint32_t n_local = c.n_kv_heads - n_full;
    b.block = blocks - 1 - index / n_local;
    n = n_full + index % n_local;
  }
  b.head = head_in_order(c, n, b.full);
  return b;
}

struct ColumnSmem {
  int32_t offsets[kOffsetsInLds];
  int32_t first[kPackedWaves], begin[kPackedWaves], last[kPackedWaves];
};
struct Columns {
  int pos, head, begin;                            // of the lane's column; begin: of its sequence
  bool valid, full;                                // a column of no sequence reads row 0 and writes nothing
  int64_t row;
  int pos_lo, pos_hi, begin_lo, begin_hi;          // of the wavefront's
  int sink, recent;
  int keys_begin, band, sink_tiles, tiles;         // of the workgroup: tiles of a full head from keys_begin on; of a local one those of the sinks
                                                   // of the first sequence, then from the first position's band on (the block's later sequences
                                                   // begin behind its first position)
  __device__ __forceinline__ int tile_key(int t) const { return t < sink_tiles ? keys_begin + t * kKeys : band + (t - sink_tiles) * kKeys; }
  __device__ __forceinline__ bool admits(int key) const {
    return key <= pos && key >= begin && (full || key - begin < sink || pos - key < recent);
  }
  // whether any, and whether all columns of the wavefront admit any, all of `n` keys from k0 on
  __device__ __forceinline__ bool any_of(int k0, int n) const {
    return k0 <= pos_hi && k0 + n > begin_lo && (full || k0 - begin_hi < sink || pos_lo - (k0 + n - 1) < recent);
  }
  __device__ __forceinline__ bool all_of(int k0, int n) const {
    return k0 + n - 1 <= pos_lo && k0 >= begin_hi && (full || k0 + n - 1 - begin_lo < sink || pos_hi - k0 < recent);
  }
};
// False: no column of the block is of a sequence.
__device__ __forceinline__ bool set_columns(const PackedCall& c, const int32_t* offsets, const ColumnBlock& b, ColumnSmem& sm, Columns& x) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t column = (uint32_t)b.block * kColumns + wave * 32 + (lane & 31);
  x.pos = (int)(column / (uint32_t)c.group);
  x.head = b.head * c.group + (int)(column - (uint32_t)x.pos * c.group);
  x.full = b.full;
  x.sink = c.sink;
  x.recent = c.recent;
  const Span span = span_of(offsets, c.n_seqs, c.tokens, x.pos);
  x.valid = span.begin >= 0;
  x.begin = x.valid ? span.begin : 0;
  x.row = x.valid ? x.pos : 0;
  x.pos_lo = min_of_lanes(x.valid ? x.pos : INT32_MAX);
  x.pos_hi = max_of_lanes(x.valid ? x.pos : -1);
  x.begin_lo = min_of_lanes(x.valid ? x.begin : INT32_MAX);
  x.begin_hi = max_of_lanes(x.valid ? x.begin : -1);
  if (lane == 0) {
    sm.first[wave] = x.pos_lo;
    sm.begin[wave] = x.begin_lo;
    sm.last[wave] = x.pos_hi;
  }
  __syncthreads();
  int first = INT32_MAX, last = -1;
  x.keys_begin = INT32_MAX;
#pragma unroll
  for (int w = 0; w < kPackedWaves; ++w) {
    first = min(first, sm.first[w]);
    x.keys_begin = min(x.keys_begin, sm.begin[w]);
    last = max(last, sm.last[w]);
  }
  if (last < 0) return false;
  x.sink_tiles = x.full ? 0 : (int)(((int64_t)min(c.sink, last + 1 - x.keys_begin) + kKeys - 1) / kKeys);
  x.band = x.full ? x.keys_begin : max(x.keys_begin + x.sink_tiles * kKeys, first - c.recent + 1);
  x.tiles = x.sink_tiles + (x.band > last ? 0 : (last - x.band) / kKeys + 1);
  return true;
}
__device__ __forceinline__ const int32_t* offsets_of(const PackedCall& c, int32_t* here) {
  if (c.n_seqs >= kOffsetsInLds) return c.offsets;
  for (int i = threadIdx.x; i <= c.n_seqs; i += kPackedThreads) here[i] = c.offsets[i];
  __syncthreads();
  return here;
}

}  // namespace rlkv
