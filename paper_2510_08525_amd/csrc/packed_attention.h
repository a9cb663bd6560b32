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
// Division of numbers below 2^31 by one that the host knows: x / d = x * mul >> (31 + shift), mul = ceil(2^(31 + shift) / d), shift = ceil(log2 d).
struct Divisor {
  uint32_t mul, shift;
  static Divisor by(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
  }
  __device__ __forceinline__ uint32_t of(uint32_t x) const { return (uint32_t)(((uint64_t)x * mul) >> (31 + shift)); }
};
struct PackedCall {
  HeadRows q, k, v, out, grad_out, grad_q, grad_k, grad_v;
  float* lse;                       // [n_q_heads][tokens]
  float* delta;                     // the same (gradient only); set by the launch
  PackedPlan* plan;         // gradient only; set by the launch
  float* slots;                     // the same
  void* workspace;                  // gradient only
  const int32_t* offsets;           // [n_seqs + 1]
  int32_t n_seqs, tokens, n_q_heads, n_kv_heads, group;
  int32_t n_full;                   // KV heads that are
  Divisor by_group, by_full, by_local;      // the numbers of query heads of a KV head, of full and of local KV heads (1 where there are none)
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
__device__ __forceinline__ Span clamped(int b, int e, int position, int tokens) {
  return {b < 0 ? 0 : b > position ? position : b, e > tokens ? tokens : e > position ? e : position + 1};
}
// The offsets as a wavefront has them: up to 63 sequences in its lanes, one turn of memory for everything that is asked of them; more stay in memory.
struct Offsets {
  const int32_t* p;
  int32_t n_seqs, tokens, lanes;
  int32_t first, last;                         // offsets[0], offsets[n_seqs]
  __device__ __forceinline__ explicit Offsets(const PackedCall& c) : p(c.offsets), n_seqs(c.n_seqs), tokens(c.tokens) {
    const int lane = threadIdx.x & 63;
    if (n_seqs < 64) {
      lanes = p[lane < n_seqs ? lane : n_seqs];
      first = __builtin_amdgcn_readlane(lanes, 0);
      last = __builtin_amdgcn_readlane(lanes, n_seqs);
    } else {
      first = p[0];
      last = p[n_seqs];
    }
  }
  // of a position that is the same in all lanes
  __device__ __forceinline__ Span of(int position) const {
    const int lane = threadIdx.x & 63;
    if (position >= tokens) return {-1, -1};
    if (n_seqs < 64) {
      const int at = __popcll(__ballot(lane <= n_seqs && lanes <= position));      // the first offset behind the position
      if (at <= 0 || at > n_seqs) return {-1, -1};
      return clamped(__builtin_amdgcn_readlane(lanes, at - 1), __builtin_amdgcn_readlane(lanes, at), position, tokens);
    }
    // the first offset behind the position is in [from, to]; 64 are looked at at a time (unsigned: places past the last one may be beyond 2^31)
    uint32_t from = 0, to = (uint32_t)n_seqs + 1;
    while (from < to) {
      const uint32_t each = (to - from + 63) / 64, at = from + (lane + 1) * each - 1;
      const uint32_t below = __popcll(__ballot(at < to && p[at < to ? at : from] <= position));      // (not decreasing: the first ones)
      from += below * each;
      to = min(to, from + each - 1);
    }
    if (from == 0 || from > (uint32_t)n_seqs) return {-1, -1};
    return clamped(p[from - 1], p[from], position, tokens);
  }
  // Positions that ascend over the lanes (over the first 32 of them, the others have the same again): each lane's own span, by as many turns as there are
  // sequences among them.
  __device__ __forceinline__ Span of_lane(int position) const {
    Span mine = {-1, -1};
    const int top = __builtin_amdgcn_readlane(position, 31);
    int at = __builtin_amdgcn_readlane(position, 0);
    while (at <= top) {
      const Span s = of(at);
      if (s.begin < 0) {                         // in front of the first sequence, or behind the last one
        if (first <= at) break;
        at = first;
        continue;
      }
      if (position >= at && position < s.end) mine = s;
      at = s.end;
    }
    return mine;
  }
};

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

__device__ __forceinline__ uint32_t two_bf16(float a, float b) {      // rounded to nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Rows in LDS, 16 units of 16 bytes each: blocks of 8 rows x 8 units (1 KiB).  Where a unit is, is a sum of what the lane and what the instruction says, so
// the reads of a tile have one to four address registers (with the units of a row permuted by its number, 24 of them, the gradient's second kernel
// kept its keys outside the registers).
//   kQuads  in a block quads of units, in a quad the rows, every fourth row's quad permuted: the 16 rows of which 16 lanes read the same unit at a time,
//           and the 4 rows x 4 units of which 32 lanes read 8 bytes each transposed, lie in banks of their own
//   kPairs  in a block pairs of units, in a pair the rows: half of the reads' time is conflicts.  Yet the forward kernel is the faster with it, for
//           reasons that its counters do not tell (16384 tokens of 32 / 8 heads 1893 us and 1990 with quads on one machine), and the gradient's slower
//           (2 x 8192 2415 us and 2227)
enum Layout { kQuads, kPairs };
template <Layout L>
__device__ __forceinline__ int unit_at(int row, int unit) {
  if (L == kQuads) return (row >> 3) * 128 + (unit >> 2) * 32 + (row & 7) * 4 + ((unit ^ (row >> 2)) & 3);
  return (row >> 3) * 128 + (unit >> 1) * 16 + (row & 7) * 2 + (unit & 1);
}
// Operand of 32 rows for the k's 16 step .. + 15 as they stand (A: rows of a tile in LDS); row0 a multiple of 32.
template <Layout L>
__device__ __forceinline__ bf16x8 row_fragment(const uint4* tile, int row0, int step) {
  const int lane = threadIdx.x & 63;
  return __builtin_bit_cast(bf16x8, tile[unit_at<L>(lane & 31, 2 * (step & 1) + (lane >> 5)) + (row0 >> 3) * 128 + (step >> 2) * 64 + (step & 2) * 16]);
}
// Operand of the 32 columns 32 block .. of a tile for 16 of its rows (row0 a multiple of 16), in the order of k that a product's result has.
template <Layout L>
__device__ __forceinline__ bf16x8 transposed_fragment(const uint4* tile, int row0, int block) {
#ifdef __HIP_DEVICE_COMPILE__
  const int lane = threadIdx.x & 63;
  const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), unit = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
  const int more = (row0 >> 3) * 128 + (block >> 1) * 64 + (block & 1) * 32;
  const char* at = reinterpret_cast<const char*>(tile + more) + 8 * (lane & 1);
  union { shorts4 part[2]; bf16x8 all; } f;
  f.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLKV_LDS_PTR(shorts4, at + unit_at<L>(row, unit) * 16));
  f.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLKV_LDS_PTR(shorts4, at + unit_at<L>(row + 8, unit) * 16));
  return f.all;
#else
  return bf16x8{};
#endif
}

// 64 rows from `token` on of a head's rows, straight from memory to a tile in LDS; all WAVES wavefronts of the workgroup are at the call.  Rows from
// `tokens` on are the last one.  (Buffer loads, whose base is the same in all lanes; a row's place from it fits 32 bits.)
constexpr int kStageRows = 64;
constexpr int64_t kMostTokenStride = 1 << 24;
template <Layout L, int WAVES>
__device__ __forceinline__ void stage_rows(const HeadRows& t, int token, int head, int tokens, uint4* tile) {
#ifdef __HIP_DEVICE_COMPILE__
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const __amdgpu_buffer_rsrc_t from =
      __builtin_amdgcn_make_buffer_rsrc(t.p + (int64_t)token * t.token + (int64_t)head * t.head, 0, 0xffffffff, 0x00027000);
  const int most = tokens - 1 - token;
#pragma unroll
  for (int i = 0; i < 16 / WAVES; ++i) {
    const int block = i * WAVES + wave, row = (block >> 1) * 8 + (L == kQuads ? (lane >> 2) & 7 : (lane >> 1) & 7);
    const int unit = (block & 1) * 8 + (L == kQuads ? (lane >> 5) * 4 + ((lane ^ (row >> 2)) & 3) : (lane >> 4) * 2 + (lane & 1));
    const uint32_t at = (uint32_t)(row < most ? row : most) * (uint32_t)(t.token * 2) + unit * 16;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, RLKV_LDS_PTR(void, tile + block * 64), 16, (int)at, 0, 0, 0);
  }
#endif
}

// All of the workgroup's loads to LDS have arrived.  (The compiler makes a wavefront wait for its own before it reads them, which may be behind the
// barrier: what another wavefront reads has to be waited for in front of it.)
__device__ __forceinline__ void tile_arrived() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Order of a stretch of instructions: `first` reads of LDS, then with every matrix instruction EACH more, so that a fragment's way (some 100 clocks)
// passes behind the products in front of it.
template <int PRODUCTS, int READS, int FIRST, int EACH>
__device__ __forceinline__ void reads_ahead() {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (FIRST + i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
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
template <Layout L, typename F>
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
        const words2 two = *reinterpret_cast<const words2*>(reinterpret_cast<const char*>(tile + unit_at<L>(row0 + row, d >> 3)) + 2 * (d & 7));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][4 * g + e] += x * __uint_as_float(e & 1 ? two[e >> 1] & 0xffff0000u : two[e >> 1] << 16);
      }
  }
}

// ---- a workgroup of columns, 32 a wavefront, and the tiles of keys that it walks over ----
constexpr int kKeys = kStageRows;
constexpr int kPackedWaves = 8;      // (with four, two workgroups a compute unit, every tile is fetched twice as often: 16384 tokens 3265 us against 2006)
inline uint32_t column_blocks(const PackedCall& c, int waves) { return (uint32_t)(((int64_t)c.tokens * c.group + 32 * waves - 1) / (32 * waves)); }

// Whether a workgroup has half as many columns and each half of its wavefronts every second tile of their keys, whose sums are added up at the end: where
// that fits the card at once, and up to twice that where sequences are long, so that the longest workgroup is what the launch lasts.  Forward, us, 28 / 4
// heads, without and with: one sequence of 70 tokens 10.2 and 8.8, 333 16.6 and 13.2, 1150 35.1 and 26.6, 2100 57.3 and 48.5, eight of 130 13.3 and 11.8, two of
// 1000 33.2 and 31.5; but three of 700 27.0 and 33.7, sixteen of 100 14.2 and 18.0, one of 3000 84 and 92.  The gradient's queries:
// 333 23.1 and 17.7, 1200 52.2 and 37.2, 2300 94 and 74, six of 300 23.9 and 31.4.
// The rule sees what the host does: the buffer's rows, those behind the last sequence among them, and all sequences, empty ones too.  2100 tokens of 28 / 4 heads
// take 51 us, with two empty sequences behind them or in a buffer of 5100 rows 58 (undivided; 16 / 1 heads 42 and 56, 1100 tokens of 32 / 8 26 and 34).
inline bool keys_divided(const PackedCall& c) {
  const int64_t workgroups = (int64_t)column_blocks(c, kPackedWaves) * c.n_kv_heads;
  return workgroups <= 128 || (workgroups <= 256 && c.tokens >= (int64_t)c.n_seqs * 1000);
}

// Block and head of the launch's workgroup `index`: of all full heads the last blocks first, then of the local ones, so that the long workgroups are
// handed out first; and neighbours in the launch, which the hardware deals to the 8 XCDs in turn, are of different heads: a head's keys are then read by
// few of the L2s.
struct ColumnBlock { int block, head; bool full; };
__device__ __forceinline__ ColumnBlock column_block(const PackedCall& c, uint32_t index, uint32_t blocks) {
  ColumnBlock b;
  b.full = index < blocks * c.n_full;
  if (!b.full) index -= blocks * c.n_full;
  const uint32_t turn = b.full ? c.by_full.of(index) : c.by_local.of(index);
  b.block = blocks - 1 - turn;
  int n = index - turn * (b.full ? c.n_full : c.n_kv_heads - c.n_full);      // the n-th of its kind
  for (int w = 0;; ++w) {
    uint64_t bits = b.full ? c.full[w] : ~c.full[w];
    const int here = __popcll(bits);
    if (n >= here) {
      n -= here;
      continue;
    }
    for (; n; --n) bits &= bits - 1;
    b.head = w * 64 + __builtin_ctzll(bits);
    return b;
  }
}

struct Columns {
  int pos, head, begin;                            // of the lane's column; begin: of its sequence
  bool valid, full;                                // a column of no sequence reads row 0 and writes nothing
  int pos_lo, pos_hi, begin_lo, begin_hi;          // of the wavefront's
  int sink, recent;
  int keys_begin, band, sink_tiles, tiles;         // of the workgroup: tiles of a full head from keys_begin on; of a local one those of the sinks
                                                   // of the first sequence, then from the first position's band on (the block's later sequences
                                                   // begin behind its first position)
  __device__ __forceinline__ int tile_key(int t) const { return t < sink_tiles ? keys_begin + t * kKeys : band + (t - sink_tiles) * kKeys; }
  int64_t row;
  int mask_begin, mask_span, mask_near;            // of the lane: admitted are mask_begin + a, 0 <= a <= mask_span and (a < sink or a > mask_near)
  // (without branches; LOCAL false: of a full head)
  template <bool LOCAL>
  __device__ __forceinline__ bool admits(int key) const {
    const int a = key - mask_begin;
    const bool in = (uint32_t)a <= (uint32_t)mask_span;
    return LOCAL ? in & ((a < sink) | (a > mask_near)) : in;
  }
  __device__ __forceinline__ bool admits(int key) const { return full ? admits<false>(key) : admits<true>(key); }
  // x of the keys that are not admitted becomes `otherwise`: results of 32 keys from k0 on
  __device__ __forceinline__ void mask(floatx16& x, int k0, float otherwise) const {
    const int first = k0 + 4 * ((threadIdx.x >> 5) & 1);
    if (full) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = admits<false>(first + 8 * (r >> 2) + (r & 3)) ? x[r] : otherwise;
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = admits<true>(first + 8 * (r >> 2) + (r & 3)) ? x[r] : otherwise;
    }
  }
  // whether any, and whether all columns of the wavefront admit any, all of `n` keys from k0 on
  __device__ __forceinline__ bool any_of(int k0, int n) const {
    return k0 <= pos_hi && k0 + n > begin_lo && (full || k0 - begin_hi < sink || pos_lo - (k0 + n - 1) < recent);
  }
  __device__ __forceinline__ bool all_of(int k0, int n) const {
    return k0 + n - 1 <= pos_lo && k0 >= begin_hi && (full || k0 + n - 1 - begin_lo < sink || pos_hi - k0 < recent);
  }
};
// What a wavefront knows of its columns' positions, each of its lanes' own.  (Where offsets make no sense, so do these, but a lane's own mask is its own.)
struct Ends { int first_lane, last_lane; };
__device__ __forceinline__ Ends ends_of(bool valid) {
  const uint32_t lanes = (uint32_t)__ballot(valid);
  return {lanes ? __builtin_ctz(lanes) : -1, lanes ? 31 - __builtin_clz(lanes) : -1};
}
// False: no column of the block, 32 for each of WAVES wavefronts (the workgroup may have them several times over), is of a sequence.
template <int WAVES>
__device__ __forceinline__ bool set_columns(const PackedCall& c, const Offsets& offsets, const ColumnBlock& b, Columns& x) {
  const uint32_t from = (uint32_t)b.block * (WAVES * 32), column = from + (threadIdx.x >> 6) % WAVES * 32 + (threadIdx.x & 31);
  x.pos = (int)c.by_group.of(column);
  x.head = b.head * c.group + (int)(column - (uint32_t)x.pos * c.group);
  x.full = b.full;
  x.sink = c.sink;
  x.recent = c.recent;
  // the block's first and last position that is of a sequence, and where the first one's begins: the same in all wavefronts
  const int first = max((int)c.by_group.of(from), offsets.first);
  const int last = min(min((int)c.by_group.of(from + WAVES * 32 - 1) + 1, c.tokens), max(offsets.last, 0)) - 1;
  if (first > last) return false;
  const Span start = offsets.of(first);
  if (start.begin < 0) return false;
  x.keys_begin = start.begin;
  x.sink_tiles = x.full ? 0 : (int)(((int64_t)min(c.sink, last + 1 - x.keys_begin) + kKeys - 1) / kKeys);
  x.band = x.full ? x.keys_begin : max(x.keys_begin + x.sink_tiles * kKeys, first - c.recent + 1);
  x.tiles = x.sink_tiles + (x.band > last ? 0 : (last - x.band) / kKeys + 1);
  Span span = start;
  if (__any(x.pos < first || x.pos >= start.end)) span = offsets.of_lane(x.pos);
  x.valid = span.begin >= 0;
  x.begin = x.valid ? span.begin : 0;
  x.row = x.valid ? x.pos : 0;
  x.mask_begin = x.valid ? x.begin : INT32_MAX;      // (none)
  x.mask_span = x.valid ? x.pos - x.begin : 0;
  x.mask_near = x.mask_span - c.recent;
  const Ends e = ends_of(x.valid);
  const bool any = e.first_lane >= 0;
  x.pos_lo = any ? __builtin_amdgcn_readlane(x.pos, e.first_lane) : INT32_MAX;
  x.pos_hi = any ? __builtin_amdgcn_readlane(x.pos, e.last_lane) : -1;
  x.begin_lo = any ? __builtin_amdgcn_readlane(x.begin, e.first_lane) : INT32_MAX;
  x.begin_hi = any ? __builtin_amdgcn_readlane(x.begin, e.last_lane) : -1;
  return true;
}
// Whether any lane of the workgroup says so.  `flag`, in LDS, has been 0 since before the last barrier.
__device__ __forceinline__ bool any_of_workgroup(bool x, int32_t& flag) {
  if (__any(x) && (threadIdx.x & 63) == 0) flag = 1;
  __syncthreads();
  return flag != 0;
}

}  // namespace rlkv
