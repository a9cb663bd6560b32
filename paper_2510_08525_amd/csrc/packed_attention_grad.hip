// Gradient of the packed attention (packed_attention.hip).  With w[i][j] = exp(scale q[i] . k[j] - lse[i]) of the admitted pairs:
//
//   delta[i] = grad_out[i] . out[i]          z[i][j] = w[i][j] (grad_out[i] . v[j] - delta[i])
//   grad_q[i] = scale sum_j z[i][j] k[j]     grad_k[j] = scale sum_i z[i][j] q[i]     grad_v[j] = sum_i w[i][j] grad_out[i]
//
// Two kernels, each of which forms w and z for itself: one walks over the keys of its columns (queries) as the forward one does and leaves grad_q
// and delta, the other over the columns of its keys and leaves grad_k and grad_v, summed over the group's heads in fp32 in a fixed order.
// That is seven products where one kernel would do five, but none of them adds to memory that others add to: equal calls give equal bits.
//
// 2 x 8192 tokens, 32 / 8 heads, half of them local: 884 us for the queries (three products), 1296 for the keys (four), 28 for sums of shared keys (2208 in all, to
// 2370 over machines); seven products at the library's rate of 1.23 PFLOP/s would be 1770.  Both are bound by the matrix cores and the vector instructions between their
// products, at two wavefronts a SIMD.  12 sequences of 50 to 700, 28 / 4 heads: 58, 85 and 13 us, where a step of 64 positions takes 3 us (its products 2) and a
// workgroup's start and end 20: keys and values, the last barrier, and 256 KiB of sums each to memory (equal stretches of all steps a workgroup, several tiles
// of keys one after the other, took 134 us for 90, and 1538 for 1370).
#include <type_traits>

#include "packed_attention.h"

namespace rlkv {
namespace {

constexpr int kWaves = kPackedWaves, kThreads = 64 * kWaves;

__device__ __forceinline__ float dot_of_units(uint4 a, uint4 b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum = __builtin_fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum);
    sum = __builtin_fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), sum);
  }
  return sum;
}

// ---- the plan: what every workgroup of the second launch does ----
constexpr int kKeysHere = 32 * kWaves, kStep = kStageRows;      // keys of a workgroup, positions of a step (below)
constexpr int kMostParts = 512;           // workgroups that share keys, at most: two a compute unit
constexpr int kLeastSteps = 4, kEnoughSteps = 16;      // steps that are worth a workgroup with a slot to write and to add up where others idle; that are in any case
constexpr int kSlotFloats = 2 * kHeadDim * kKeysHere;

struct PlanItem {
  int32_t tile, head;                     // keys [256 tile, + 256) of KV head `head`
  int32_t first, end;                     // the positions that admit any of them
  int32_t step, last_step;                // of their steps the ones [step, last_step)
  int32_t slot;                           // where the sums go; -1: into the gradients
  int32_t pad;
};
struct PlanMerge { int32_t slot, parts; };      // of a tile and head: parts 0 where nothing is shared
// (behind the PackedPlan: PlanItem[tiles * heads + kMostParts], PlanMerge[tiles * heads])
__host__ __device__ inline int64_t tiles_of(int64_t tokens) { return (tokens + kKeysHere - 1) / kKeysHere; }
__device__ __forceinline__ PlanItem* items_of(PackedPlan* p) { return reinterpret_cast<PlanItem*>(p + 1); }
__device__ __forceinline__ PlanMerge* merges_of(PackedPlan* p, int64_t pairs) { return reinterpret_cast<PlanMerge*>(items_of(p) + pairs + kMostParts); }

// Steps of a part: parts have at least as many and less than twice as many, so there are at most kMostParts of them; half as many where they are short.
// (A call may have 2^45 steps, of which a tile's keys have 2^28 at most: a share of more than 2^31 divides none of them, and counts as 2^31 - 1.)
__host__ __device__ constexpr int least_steps(unsigned long long total) {
  const int64_t share = (int64_t)((total + kMostParts - 1) / kMostParts), twice = 2 * share < kEnoughSteps ? 2 * share : kEnoughSteps;
  const int64_t least = share > twice ? share : twice;
  return least > INT32_MAX ? INT32_MAX : least > kLeastSteps ? (int)least : kLeastSteps;
}
constexpr bool parts_fit(unsigned long long total) { return least_steps(total) > 1 << 28 || total / (unsigned long long)least_steps(total) <= kMostParts; }
static_assert(least_steps(0) == 4 && least_steps(512) == 4 && least_steps(2049) == 10 && least_steps(4097) == 16 && least_steps(512 * 100) == 100, "");
static_assert(parts_fit(3000) && parts_fit(1ull << 31) && parts_fit(1ull << 40) && parts_fit((1ull << 41) + (1 << 23)) && parts_fit(1ull << 45), "");

struct PlanSmem {
  unsigned long long total;
  int32_t items, slots;
};
// The positions of a tile's keys; end <= first: none.
struct TileRange { int32_t first, end; };
__device__ __forceinline__ TileRange range_of(const PackedCall& c, int tile, bool full) {
  const int32_t* offsets = c.offsets;
  const int begin = offsets[0], end = offsets[c.n_seqs];
  const int first = max(tile * kKeysHere, begin), last = min(min(tile * kKeysHere + kKeysHere, end), c.tokens) - 1;
  if (first > last) return {0, 0};
  int lo = 0, hi = c.n_seqs + 1;              // (every thread has a tile of its own)
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (offsets[mid] > last) hi = mid;
    else lo = mid + 1;
  }
  if (lo == 0 || lo > c.n_seqs) return {0, 0};
  const Span span = {min(max(offsets[lo - 1], 0), last), min(offsets[lo], c.tokens)};
  if (full || max(span.begin, first) - span.begin < c.sink || span.end - last < c.recent) return {first, span.end};
  return {first, last + c.recent};
}
__device__ __forceinline__ int steps_of(const TileRange& r, int group) {
  return r.end <= r.first ? 0 : (r.end - r.first + kStep - 1) / kStep * group;
}
// One workgroup.
__device__ void make_plan(const PackedCall& c, PlanSmem& sm) {
  const int64_t pairs = tiles_of(c.tokens) * c.n_kv_heads;
  if (threadIdx.x == 0) {
    sm.total = 0;
    sm.items = sm.slots = 0;
  }
  __syncthreads();
  auto pair = [&](int64_t i, int& tile, int& h) {
    tile = (int)(i / c.n_kv_heads);
    h = (int)(i - (int64_t)tile * c.n_kv_heads);
    return range_of(c, tile, (c.full[h >> 6] >> (h & 63)) & 1);
  };
  int tile, h;
  unsigned long long mine = 0;
  for (int64_t i = threadIdx.x; i < pairs; i += blockDim.x) mine += steps_of(pair(i, tile, h), c.group);
  atomicAdd(&sm.total, mine);
  __syncthreads();
  const int least = least_steps(sm.total);
  PlanItem* items = items_of(c.plan);
  PlanMerge* merges = merges_of(c.plan, pairs);
  // (the long ones in front of the others)
  for (int turn = 0; turn < 2; ++turn) {
    for (int64_t i = threadIdx.x; i < pairs; i += blockDim.x) {
      const TileRange r = pair(i, tile, h);
      const int steps = steps_of(r, c.group), parts = max(1, steps / least);
      if (turn == 0) merges[i] = {-1, 0};
      if (steps == 0 || (steps >= least) != (turn == 0)) continue;
      const int at = atomicAdd(&sm.items, parts), slot = parts > 1 ? atomicAdd(&sm.slots, parts) : -1;
      if (parts > 1) merges[i] = {slot, parts};
      for (int p = 0; p < parts; ++p)
        items[at + p] = {tile, h, r.first, r.end, (int)((int64_t)steps * p / parts), (int)((int64_t)steps * (p + 1) / parts), parts > 1 ? slot + p : -1, 0};
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) c.plan->items = sm.items;
}

// ---- queries ------------------------------------------------------------------------------------------------------------------
// SPLIT 2: the keys are divided between the halves of the workgroup (keys_divided).
template <int WAVES, int SPLIT>
__global__ __launch_bounds__(64 * WAVES) void packed_grad_q_kernel(PackedCall c, uint32_t blocks) {
  constexpr int kColumnWaves = WAVES / SPLIT;
  __shared__ uint4 t0[SPLIT][2][kKeys * 16], t1[SPLIT][2][kKeys * 16];      // keys, values
  __shared__ PlanSmem plan;
  const int half = (threadIdx.x >> 5) & 1, part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kColumnWaves : 0;
  if (blockIdx.x == 0) {                                     // (the launch's first workgroup plans the next launch)
    make_plan(c, plan);
    return;
  }
  __shared__ int32_t lost;
  const Offsets offsets(c);
  const ColumnBlock block = column_block(c, blockIdx.x - 1, blocks);
  Columns x;
  if (!set_columns<kColumnWaves>(c, offsets, block, x)) return;
  if (threadIdx.x == 0) lost = 0;

  bf16x8 q[8], g[8];
  uint4 out[8];
  const int64_t stat = (int64_t)x.head * c.tokens + x.row;
  const float lse = c.lse[stat] * kLog2e;
  {
    const uint16_t* q_row = c.q.p + x.row * c.q.token + x.head * c.q.head + 8 * half;
    const uint16_t* g_row = c.grad_out.p + x.row * c.grad_out.token + x.head * c.grad_out.head + 8 * half;
    const uint16_t* o_row = c.out.p + x.row * c.out.token + x.head * c.out.head + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      g[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(g_row + 16 * s));
      out[s] = *reinterpret_cast<const uint4*>(o_row + 16 * s);
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q_row + 16 * s));
  }
  const float scale = c.scale * kLog2e;
  auto ask = [&](auto odd, int t) {
    constexpr int kOdd = decltype(odd)::value;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i) {
      if (i > 0 && t + i >= x.tiles) break;
      stage_rows<kQuads, WAVES>(c.k, x.tile_key(t + i), block.head, c.tokens, kOdd ? t1[i][0] : t0[i][0]);
      stage_rows<kQuads, WAVES>(c.v, x.tile_key(t + i), block.head, c.tokens, kOdd ? t1[i][1] : t0[i][1]);
    }
  };

  // (while the first tile is under way)
  ask(std::integral_constant<int, 0>{}, 0);
  float delta = 0.f;
#pragma unroll
  for (int s = 0; s < 8; ++s) delta += dot_of_units(__builtin_bit_cast(uint4, g[s]), out[s]);
  delta = sum_of_halves(delta);
  if (x.valid && half == 0 && part == 0) c.delta[stat] = delta;

  floatx16 dq[4];
  auto walk = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
#pragma unroll
    for (int b = 0; b < 4; ++b) clear(dq[b]);
    if (kCareful) ask(std::integral_constant<int, 0>{}, 0);
    auto step = [&](auto odd, int t) {
      constexpr int kOdd = decltype(odd)::value;
      const uint4 *kt = kOdd ? t1[part][0] : t0[part][0], *vt = kOdd ? t1[part][1] : t0[part][1];
      tile_arrived();
      if (t + SPLIT < x.tiles) ask(std::integral_constant<int, 1 - kOdd>{}, t + SPLIT);
      if (part > 0 && t + part >= x.tiles) return;
#pragma unroll
      for (int b = 0; b < kKeys; b += 32) {
        const int key = x.tile_key(t + part) + b;
        if (!x.any_of(key, 32)) continue;
        const bool all = x.all_of(key, 32);
        floatx16 w, z;
        clear(w);
        clear(z);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          w = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment<kQuads>(kt, b, s), q[s], w, 0, 0, 0);
          z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment<kQuads>(vt, b, s), g[s], z, 0, 0, 0);
        }
        reads_ahead<16, 16, 4, 1>();
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(w[r], scale, -lse)) * (z[r] - delta);
        if (!all) x.mask(z, key, 0.f);
        if (kCareful && !all) {
          admitted_products<kQuads>(kt, b, z, dq, [&](int r) { return x.admits(key + r); });
        } else {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const bf16x8 p = weights_fragment(z, s);
#pragma unroll
            for (int d = 0; d < 4; ++d) dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment<kQuads>(kt, b + 16 * s, d), p, dq[d], 0, 0, 0);
          }
          reads_ahead<8, 16, 6, 2>();
        }
      }
    };
    int t = 0;
    for (; t + SPLIT < x.tiles; t += 2 * SPLIT) {
      step(std::integral_constant<int, 0>{}, t);
      step(std::integral_constant<int, 1>{}, t + SPLIT);
    }
    if (t < x.tiles) step(std::integral_constant<int, 0>{}, t);
  };
  walk(std::false_type{});
  if (any_of_workgroup(x.valid && zero_or_nan(dq) != 0.f, lost)) walk(std::true_type{});
  if (SPLIT > 1) {
    // the second half's sums to the first, in the tiles' place
    float4* sums = reinterpret_cast<float4*>(t0);
    const int at = threadIdx.x % (64 * kColumnWaves);
    __syncthreads();
    if (part == 1) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        sums[i * 64 * kColumnWaves + at] = make_float4(dq[i >> 2][4 * (i & 3)], dq[i >> 2][4 * (i & 3) + 1], dq[i >> 2][4 * (i & 3) + 2], dq[i >> 2][4 * (i & 3) + 3]);
    }
    __syncthreads();
    if (part == 1) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float4 y = sums[i * 64 * kColumnWaves + at];
      dq[i >> 2][4 * (i & 3)] += y.x;
      dq[i >> 2][4 * (i & 3) + 1] += y.y;
      dq[i >> 2][4 * (i & 3) + 2] += y.z;
      dq[i >> 2][4 * (i & 3) + 3] += y.w;
    }
  }
  store_rows(c.grad_q.p + x.row * c.grad_q.token + x.head * c.grad_q.head, dq, c.scale, x.valid);
}

// ---- keys and values ----------------------------------------------------------------------------------------------------------
// A workgroup has 256 keys, 32 a wavefront and one a lane (both halves of the wavefront: the same), and walks over the positions that admit any of
// them, 64 of one query head of the group at a time, a head after the other.  Key j is admitted to the positions j <= i < limit: the end of its
// sequence, or of a local head's key that is no sink j + recent if that is less.
//
// How many steps that is differs by a thousand between the keys of a launch (the first keys of a long sequence, the sinks of a local head,
// short sequences), so the launch in front plans: a workgroup is given at most some 2 / 512 of all steps, and where keys have more they are
// divided among workgroups that leave their sums in slots of the workspace, which a third launch adds up in the order of the steps.

// Sums of a workgroup in its slot, and the way back: piece (which of the 32 float4 of a lane) after piece, lane after lane.
__device__ __forceinline__ float* slot_piece(float* slots, int slot, int piece, int thread) {
  return slots + (int64_t)slot * kSlotFloats + ((int64_t)piece * kThreads + thread) * 4;
}

__global__ __launch_bounds__(kThreads) void packed_grad_kv_kernel(PackedCall c) {
  // (objects of their own, and the slot of a step known at compile time: else reads of one tile would wait for the loads of the next)
  __shared__ uint4 t0[2][kStep * 16], t1[2][kStep * 16];      // queries, gradients
  __shared__ uint4 values[kKeysHere * 16];
  __shared__ float minus_lse[2][kStep], minus_delta[2][kStep];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  __shared__ int32_t lost;
  if ((int)blockIdx.x >= c.plan->items) return;
  const Offsets offsets(c);
  if (threadIdx.x == 0) lost = 0;
  const PlanItem item = items_of(c.plan)[blockIdx.x];
  const int h = item.head, group = c.group;
  const bool full = (c.full[h >> 6] >> (h & 63)) & 1;
  const int at = item.tile * kKeysHere + (threadIdx.x >> 6) * 32 + (lane & 31);
  const Span span = offsets.of_lane(at);
  const bool valid = span.begin >= 0;
  const int key = valid ? at : 0;                                       // (a key of no sequence: nothing is admitted, nothing written)
  int limit = !valid ? 0 : full || key - span.begin < c.sink || span.end - key < c.recent ? span.end : key + c.recent;
  limit = min(limit, item.end);
  const uint32_t width = valid ? max(limit - key, 0) : 0;
  // of the wavefront: keys ascend; the least and the largest limit over its valid lanes
  const Ends ends = ends_of(valid);
  const int key_lo = ends.first_lane >= 0 ? __builtin_amdgcn_readlane(key, ends.first_lane) : INT32_MAX;
  const int key_hi = ends.first_lane >= 0 ? __builtin_amdgcn_readlane(key, ends.last_lane) : -1;
  int limit_lo = valid ? limit : INT32_MAX, limit_hi = valid ? limit : -1;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    limit_lo = min(limit_lo, __shfl_xor(limit_lo, d));
    limit_hi = max(limit_hi, __shfl_xor(limit_hi, d));
  }
  limit_lo = __builtin_amdgcn_readfirstlane(limit_lo);
  limit_hi = __builtin_amdgcn_readfirstlane(limit_hi);

  // Keys stay in registers; values, which would leave no room to read ahead, in LDS.
#pragma unroll
  for (int i = 0; i < kKeysHere; i += kStageRows)
    if (item.tile * kKeysHere + i < c.tokens) stage_rows<kQuads, kWaves>(c.v, item.tile * kKeysHere + i, h, c.tokens, values + i * 16);
  bf16x8 k[8];
  {
    const uint16_t* k_row = c.k.p + (int64_t)key * c.k.token + h * c.k.head + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) k[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(k_row + 16 * s));
  }
  const uint4* own_values = values + (threadIdx.x >> 6) * 32 * 16;

  const int per_head = (item.end - item.first + kStep - 1) / kStep;      // steps of a query head
  const float scale = c.scale * kLog2e, inv_scale = 1.f / c.scale;
  // the step that is asked for next: query head and first position
  int next_head, next_pos;
  auto ask = [&](auto odd) {
    constexpr int kOdd = decltype(odd)::value;
    stage_rows<kQuads, kWaves>(c.q, next_pos, next_head, c.tokens, kOdd ? t1[0] : t0[0]);
    stage_rows<kQuads, kWaves>(c.grad_out, next_pos, next_head, c.tokens, kOdd ? t1[1] : t0[1]);
    if (threadIdx.x < kStep) {
      const int64_t row = (int64_t)next_head * c.tokens + min(next_pos + (int)threadIdx.x, c.tokens - 1);
      minus_lse[kOdd][threadIdx.x] = -c.lse[row] * inv_scale;
      minus_delta[kOdd][threadIdx.x] = -c.delta[row];
    }
    next_pos += kStep;
    if (next_pos >= item.end) {
      next_pos = item.first;
      ++next_head;
    }
  };

  floatx16 dk[4], dv[4];
  auto walk = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      clear(dk[b]);
      clear(dv[b]);
    }
    next_head = h * group + item.step / per_head;
    next_pos = item.first + item.step % per_head * kStep;
    int pos = next_pos;
    ask(std::integral_constant<int, 0>{});
    auto step = [&](auto odd, bool more) {
      constexpr int kOdd = decltype(odd)::value;
      const uint4 *qt = kOdd ? t1[0] : t0[0], *gt = kOdd ? t1[1] : t0[1];
      tile_arrived();
      if (more) ask(std::integral_constant<int, 1 - kOdd>{});
#pragma unroll
      for (int sub = 0; sub < kStep; sub += 32) {
        const int p0 = pos + sub;
        if (p0 + 31 < key_lo || p0 >= limit_hi) continue;
        const bool all = p0 >= key_hi && p0 + 32 <= limit_lo;
        floatx16 x, y;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int col = sub + 8 * (r >> 2) + 4 * half + (r & 3);
          x[r] = minus_lse[kOdd][col];
          y[r] = minus_delta[kOdd][col];
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment<kQuads>(qt, sub, s), k[s], x, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment<kQuads>(gt, sub, s), row_fragment<kQuads>(own_values, 0, s), y, 0, 0, 0);
        }
        reads_ahead<16, 24, 5, 2>();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          x[r] = __builtin_amdgcn_exp2f(x[r] * scale);
          y[r] *= x[r];
        }
        if (!all) {
          const uint32_t from = p0 + 4 * half - key;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (from + (8 * (r >> 2) + (r & 3)) >= width) x[r] = y[r] = 0.f;
        }
        if (kCareful && !all) {
          auto admits = [&](int col) { return (uint32_t)(p0 + col - key) < width; };
          admitted_products<kQuads>(gt, sub, x, dv, admits);
          admitted_products<kQuads>(qt, sub, y, dk, admits);
        } else {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const bf16x8 w = weights_fragment(x, s), z = weights_fragment(y, s);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment<kQuads>(gt, sub + 16 * s, d), w, dv[d], 0, 0, 0);
              dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment<kQuads>(qt, sub + 16 * s, d), z, dk[d], 0, 0, 0);
            }
          }
          reads_ahead<16, 32, 6, 2>();
        }
      }
      pos += kStep;
      if (pos >= item.end) pos = item.first;
    };
    int t = item.step;
    for (; t + 1 < item.last_step; t += 2) {
      step(std::integral_constant<int, 0>{}, true);
      step(std::integral_constant<int, 1>{}, t + 2 < item.last_step);
    }
    if (t < item.last_step) step(std::integral_constant<int, 0>{}, false);
  };
  walk(std::false_type{});
  // (a weight of 0 does not keep an infinity or a NaN of a row that is not admitted out of the products)
  if (any_of_workgroup(valid && (zero_or_nan(dk) != 0.f || zero_or_nan(dv) != 0.f), lost)) walk(std::true_type{});
  if (item.slot >= 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      *reinterpret_cast<float4*>(slot_piece(c.slots, item.slot, i, threadIdx.x)) =
          make_float4(dk[i >> 2][4 * (i & 3)], dk[i >> 2][4 * (i & 3) + 1], dk[i >> 2][4 * (i & 3) + 2], dk[i >> 2][4 * (i & 3) + 3]);
      *reinterpret_cast<float4*>(slot_piece(c.slots, item.slot, 16 + i, threadIdx.x)) =
          make_float4(dv[i >> 2][4 * (i & 3)], dv[i >> 2][4 * (i & 3) + 1], dv[i >> 2][4 * (i & 3) + 2], dv[i >> 2][4 * (i & 3) + 3]);
    }
    return;
  }
  store_rows(c.grad_k.p + (int64_t)key * c.grad_k.token + h * c.grad_k.head, dk, c.scale, valid);
  store_rows(c.grad_v.p + (int64_t)key * c.grad_v.token + h * c.grad_v.head, dv, 1.f, valid);
}

// The slots of keys that workgroups shared, added up in the order of their steps: four pieces of a lane a workgroup.
__global__ __launch_bounds__(kThreads) void packed_grad_sum_kernel(PackedCall c) {
  const int64_t pairs = tiles_of(c.tokens) * c.n_kv_heads;
  const PlanMerge merge = merges_of(c.plan, pairs)[blockIdx.x];
  if (merge.parts == 0) return;
  const int tile = blockIdx.x / c.n_kv_heads, h = blockIdx.x % c.n_kv_heads, lane = threadIdx.x & 63;
  float4 sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = *reinterpret_cast<const float4*>(slot_piece(c.slots, merge.slot, blockIdx.y * 4 + i, threadIdx.x));
  for (int p = 1; p < merge.parts; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(slot_piece(c.slots, merge.slot + p, blockIdx.y * 4 + i, threadIdx.x));
      sum[i].x += x.x;
      sum[i].y += x.y;
      sum[i].z += x.z;
      sum[i].w += x.w;
    }
  const int key = tile * kKeysHere + (threadIdx.x >> 6) * 32 + (lane & 31);
  if (Offsets(c).of_lane(key).begin < 0) return;
  const HeadRows& to = blockIdx.y < 4 ? c.grad_k : c.grad_v;
  const float scale = blockIdx.y < 4 ? c.scale : 1.f;
  uint16_t* row = to.p + (int64_t)key * to.token + h * to.head + 32 * (blockIdx.y & 3) + 4 * (lane >> 5);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const words2 w = {two_bf16(sum[i].x * scale, sum[i].y * scale), two_bf16(sum[i].z * scale, sum[i].w * scale)};
    *reinterpret_cast<words2*>(row + 8 * i) = w;
  }
}

}  // namespace

// The workspace: delta, the plan, the slots.
struct GradSpace {
  size_t delta, plan, slots, bytes;
};
static GradSpace grad_space(int64_t tokens, int64_t n_q_heads, int64_t n_kv_heads) {
  const int64_t pairs = tiles_of(tokens) * n_kv_heads, group = n_q_heads / n_kv_heads;
  auto align = [](size_t x) { return (x + 255) / 256 * 256; };
  GradSpace s;
  s.delta = 0;
  s.plan = align((size_t)(tokens * n_q_heads) * sizeof(float));
  s.slots = s.plan + align(sizeof(PackedPlan) + (size_t)(pairs + kMostParts) * sizeof(PlanItem) + (size_t)pairs * sizeof(PlanMerge));
  // (parts have kLeastSteps steps at least, of which a pair has one for each head and 64 positions at most; one of fewer than two parts' has no slot)
  const int64_t of_pair = (tokens + kStep - 1) / kStep * group, steps = pairs * of_pair, parts = of_pair < 2 * kLeastSteps ? 0 : steps / kLeastSteps;
  s.bytes = s.slots + (size_t)(parts < kMostParts ? parts : kMostParts) * kSlotFloats * sizeof(float);
  return s;
}
size_t packed_grad_workspace(int tokens, int n_q_heads, int n_kv_heads) { return grad_space(tokens, n_q_heads, n_kv_heads).bytes; }

hipError_t launch_packed_attention_grad(PackedCall call, hipStream_t stream) {
  const GradSpace space = grad_space(call.tokens, call.n_q_heads, call.n_kv_heads);
  char* work = static_cast<char*>(call.workspace);
  call.delta = reinterpret_cast<float*>(work + space.delta);
  call.plan = reinterpret_cast<PackedPlan*>(work + space.plan);
  call.slots = reinterpret_cast<float*>(work + space.slots);
  const int64_t pairs = tiles_of(call.tokens) * call.n_kv_heads;
  const uint32_t blocks = column_blocks(call, kWaves), few = column_blocks(call, kWaves / 2);
  if (keys_divided(call)) packed_grad_q_kernel<kWaves, 2><<<few * (uint32_t)call.n_kv_heads + 1, kThreads, 0, stream>>>(call, few);
  else packed_grad_q_kernel<kWaves, 1><<<blocks * (uint32_t)call.n_kv_heads + 1, kThreads, 0, stream>>>(call, blocks);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int64_t parts = (int64_t)(space.bytes - space.slots) / (int64_t)(kSlotFloats * sizeof(float));
  packed_grad_kv_kernel<<<dim3((uint32_t)(pairs + parts)), kThreads, 0, stream>>>(call);
  err = hipGetLastError();
  if (err != hipSuccess || parts == 0) return err;
  packed_grad_sum_kernel<<<dim3((uint32_t)pairs, 8), kThreads, 0, stream>>>(call);
  return hipGetLastError();
}

}  // namespace rlkv
