// Log probabilities of given tokens, entropy, log-sum-exp and the most likely tokens of rows of logits, in one read of them; and the
// gradient of log probabilities and entropies.
//
// With l the logits and c = scale * log2(e), per row:
//   m = max l,  s = sum 2^(c (l - m)),  t = sum 2^(c (l - m)) c (l - m)          (running: a larger maximum rescales s and t)
//   lse = scale m + ln s      log p(token) = scale (l - m) - ln s      entropy = lse - sum p x = ln s - ln 2 * t / s
//   d logit_i = scale * (g_lp (i == token) - p_i (g_lp + g_h (log p_i + entropy)))
// The maximum is that of the logits themselves and subtracted before the scaling: masks of the type's lowest value do not overflow, and
// far from 0 nothing is lost.  Exponents stay in the base 2 until the end.  A thread keeps its own maximum, so nothing crosses lanes inside
// a row; a masked logit (-inf) has weight 0 and its exponent, -inf, is replaced by a finite one before it is multiplied by
// that; a row of nothing else has lse -inf.
//
// Most likely tokens: the key of a logit is (value, lowest index first) in 64 bits.  A workgroup works through its columns in chunks that
// it holds in registers, and collects in LDS what may be among the k best: what reaches the k-th best known so far.  Where
// many threads have something that does, that is raised to the k-th largest of the threads' maxima, which k logits reach (20 of 4096
// random ones let about 22 through).  The list is ranked by counting when it
// has grown to some times k, which raises what the next chunks have to reach, and at the end.  A chunk that lets through
// more than the list holds (ties, masks) is searched maximum by maximum.
// Few rows are split over workgroups, whose partial results a second kernel joins in a fixed order.
// Bound: HBM; 6 or 7 vector instructions and an exponential a logit are not far behind.
#include <type_traits>

#include "token_ops.h"

namespace rlkv {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256;
constexpr int kPieces = 8, kFewPieces = 2;              // pieces of eight logits of a thread in a chunk, of many rows and of few
constexpr int kList = 1024;                             // candidates a workgroup ranks at once
constexpr int kSomeMore = 4;                            // threads with candidates, in k, that a chunk may have before it raises the bound
constexpr int kMostSplits = 64;                         // workgroups a row is split over: a lane each when they are joined
constexpr float kMaskedLse = -1e30f;
constexpr float kLow = -256.f;                          // in the place of exponents so low that their weight is 0

struct Stats { float m, s, t; };                        // maximum of the logits, sum, weighted sum (exponents of base 2)

// Weighted by 2^(c (own maximum - m)); m is at least that maximum.
__device__ __forceinline__ Stats rescaled(const Stats& v, float m, float scale2) {
  if (m == -INFINITY) return v;                                 // (sums of zeros; a NaN stays one)
  const float d = (v.m - m) * scale2, w = __builtin_amdgcn_exp2f(d);
  return Stats{m, v.s * w, (v.t + v.s * fmaxf(d, kLow)) * w};
}
__device__ __forceinline__ Stats stats_of_wave(Stats v, float scale2) {
  v = rescaled(v, max_of_wave(v.m), scale2);
  return Stats{max_of_wave(v.m), sum_of_wave(v.s), sum_of_wave(v.t)};
}

// Order of logits as unsigned numbers: larger values first, NaN above all, and nothing at the end of the range, so that no key is ~0.
constexpr uint32_t kNanOrder = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return kNanOrder;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);        // (-0 and 0 are equal)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  if (order == kNanOrder) return __builtin_nanf("");
  return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
// (value, index) as one key; 0 is below every key of a logit
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ uint64_t max_of_wave(uint64_t x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint64_t y = (uint64_t)__shfl_xor((uint32_t)(x >> 32), m) << 32 | (uint32_t)__shfl_xor((uint32_t)x, m);
    x = y > x ? y : x;
  }
  return x;
}
// The k-th largest (k from 1) of N values of 16 bits a lane.
template <int N>
__device__ __forceinline__ uint32_t kth_of_wave(const uint32_t (&upper)[N], int k) {
  constexpr int kBits = N == 1 ? 2 : 1;                         // (bits a step: of one value a lane, three counts side by side take no longer)
  uint32_t kth = 0;
#pragma unroll
  for (int bit = 16 - kBits; bit >= 0; bit -= kBits) {
    uint32_t digit = 0;
#pragma unroll
    for (uint32_t t = 1; t < 1u << kBits; ++t) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) n += __popcll(__ballot(upper[i] >= (kth | t << bit)));
      if (n >= k) digit = t;
    }
    kth |= digit << bit;
  }
  return kth;
}
// An order as a value that it and larger ones reach.
__device__ __forceinline__ float bound_of(uint32_t order) { return order < 0x00800000u ? -INFINITY : value_of(order); }

// Inclusive prefix sums over the wavefront.
__device__ __forceinline__ int prefix_of_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);        // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);        // row_bcast:15, :31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

struct TopLds {
  uint64_t best[kMostTop];          // the best so far, largest first, 0 = none
  alignas(16) uint64_t list[kList + 8];      // candidates, the best so far first, and room for zeros behind them
  uint64_t wave_best[kThreads / 64];
  alignas(8) uint16_t most[64][kThreads / 64];      // upper halves of the orders of the lanes' largest logits
  int32_t some[kThreads / 64];
  int32_t n;
};
// Nothing yet.  (The next barrier is before the first use.)
__device__ __forceinline__ void clear_list(TopLds& lds) {
  if (threadIdx.x < kMostTop) lds.best[threadIdx.x] = 0;
  if (threadIdx.x == 0) lds.n = 0;
}

// list[0, n) (distinct keys and zeros, n <= kList, all threads past a barrier) -> the k largest of them into best, in order.  (Equal zeros
// take one place, and those behind it hold zeros already: what was there before is in the list too.)
__device__ void rank_list(TopLds& lds, int n, int k) {
  if (threadIdx.x < 8) lds.list[n + threadIdx.x] = 0;            // (eight keys a turn, all of them on their way at once)
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t x = lds.list[i];
    int rank = 0;
    for (int o = 0; o < n; o += 8) {
      uint64_t y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) y[u] = lds.list[o + u];
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += y[u] > x;
    }
    if (rank < k) lds.best[rank] = x;
  }
  __syncthreads();
}
// The list is the best so far and nothing else.
__device__ void restart_list(TopLds& lds, int k) {
  if ((int)threadIdx.x < k) lds.list[threadIdx.x] = lds.best[threadIdx.x];
  if (threadIdx.x == 0) lds.n = k;
  __syncthreads();
}

template <typename T> __device__ __forceinline__ float value_at(const Piece<T>& p, int i);
template <> __device__ __forceinline__ float value_at<uint16_t>(const Piece<uint16_t>& p, int i) {
  return __uint_as_float(i & 1 ? p.w[i >> 1] & 0xffff0000u : p.w[i >> 1] << 16);
}
template <> __device__ __forceinline__ float value_at<float>(const Piece<float>& p, int i) { return i < 4 ? p.a[i] : p.b[i - 4]; }

// Brings the chunk that starts at column `first` (valid: below `last`), in x, into the list.  most: a lane's largest logit of the chunk;
// odd: the lane has met a NaN or an infinity; bound: what a logit has to reach to be among the k best, the same in all lanes; row: the logits again.
// n_list: what the list holds.
template <typename T, int PIECES>
__device__ void top_of_chunk(TopLds& lds, const Piece<T> (&x)[PIECES], const T* row, int first, int last, int k, float most, bool odd,
                             float& bound, int& n_list) {
  constexpr int kWaves = kThreads / 64;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n_before = n_list;
  const uint64_t some = __ballot(most >= bound);
  const bool any_odd = __ballot(odd) != 0;
  lds.most[lane][wave] = (uint16_t)(order_of(most) >> 16);
  if (lane == 0) lds.some[wave] = __popcll(some);
  __syncthreads();
  int n_some = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) n_some += __builtin_amdgcn_readfirstlane(lds.some[w]);
  if (n_some > kSomeMore * k) {
    uint32_t upper[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) upper[w] = lds.most[lane][w];
    bound = fmaxf(bound, bound_of(kth_of_wave(upper, k) << 16));
  }
  if (some != 0 || any_odd) {
    // Which logits of the lane pass (a NaN does), then their keys: one counter update a wavefront.
    uint64_t pass = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) bits |= value_at(x[p], i) < bound ? 0u : 1u << i;
      const int col = first + (p * kThreads + tid) * 8;
      if (col + 8 > last) bits &= col < last ? (1u << (last - col)) - 1u : 0u;
      pass |= (uint64_t)bits << (8 * p);
    }
    const int mine = __popcll(pass), up_to = prefix_of_wave(mine), all = __builtin_amdgcn_readlane(up_to, 63);
    int at = 0;
    if (all != 0 && lane == 0) at = atomicAdd(&lds.n, all);
    at = __builtin_amdgcn_readfirstlane(at) + up_to - mine;
    for (; pass != 0 && at < kList; pass &= pass - 1, ++at) {          // (from the row itself: no code per logit)
      const int bit = __builtin_ctzll(pass), col = first + ((bit >> 3) * kThreads + tid) * 8 + (bit & 7);
      lds.list[at] = key_of(one_value(row[col]), col);
    }
  }
  __syncthreads();
  const int n = n_list = lds.n;
  if (n <= 4 * k + 32) return;
  if (n <= kList) {
    rank_list(lds, n, k);
  } else {
    // Maximum by maximum, each below the one before, of this chunk and of what was in the list before it.
    __syncthreads();
    uint64_t below = ~0ull;
    for (int r = 0; r < k; ++r) {
      uint64_t best = 0;
      for (int i = tid; i < n_before; i += kThreads) {
        const uint64_t key = lds.list[i];
        if (key < below && key > best) best = key;
      }
      const int end = first + kThreads * PIECES * 8 < last ? first + kThreads * PIECES * 8 : last;
      for (int col = first + tid; col < end; col += kThreads) {
        const uint64_t key = key_of(one_value(row[col]), col);
        if (key < below && key > best) best = key;
      }
      best = max_of_wave(best);
      if (lane == 0) lds.wave_best[wave] = best;
      __syncthreads();
      best = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) best = lds.wave_best[w] > best ? lds.wave_best[w] : best;
      if (tid == 0) lds.best[r] = best;
      below = best;
      __syncthreads();
    }
  }
  // (Later columns do not displace an equal logit: more than the k-th best's value is needed.  0: there are fewer than k yet.)
  const uint32_t worst = (uint32_t)(lds.best[k - 1] >> 32);
  bound = worst == 0 ? -INFINITY : worst >= order_of(INFINITY) ? INFINITY : value_of(worst + 1);
  restart_list(lds, k);
  n_list = k;
}

__device__ __forceinline__ Stats stats_of_block(Stats v, Stats (&parts)[kThreads / 64], float scale2) {
  v = stats_of_wave(v, scale2);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = parts[0].m;
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) m = fmaxf(m, parts[w].m);
  v = Stats{m, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const Stats part = rescaled(parts[w], m, scale2);
    v.s += part.s;
    v.t += part.t;
  }
  return v;
}

// What a row's results are made of: in the workspace, per row and split.
__device__ __forceinline__ Stats* part_stats(const LogprobCall& c, int64_t at) { return static_cast<Stats*>(c.workspace) + at; }
__device__ __forceinline__ uint64_t* part_best(const LogprobCall& c, int64_t at) {
  const size_t stats = ((size_t)c.rows * c.splits * sizeof(Stats) + 7) / 8 * 8;
  return reinterpret_cast<uint64_t*>(static_cast<char*>(c.workspace) + stats) + at * c.top;
}

// The logit of the row's token (thread 0, where it is asked for).
template <typename T>
__device__ __forceinline__ float logit_of(const LogprobCall& c, int row, int token) {
  return token >= 0 && token < c.vocab ? one_value((static_cast<const T*>(c.logits) + row * c.stride)[token]) : 0.f;
}
template <bool TOP>
__device__ void finish_row(const LogprobCall& c, int row, const Stats& v, const uint64_t* best, int token, float logit) {
  const float scale2 = c.scale * kLog2e, log2_s = log2f(v.s);
  const bool empty = v.s == 0.f;                                // (nothing but masked logits)
  auto logprob = [&](float x) { return empty ? -INFINITY : kLn2 * ((x - v.m) * scale2 - log2_s); };
  if (threadIdx.x == 0) {
    if (c.lse) c.lse[row] = empty ? -INFINITY : __builtin_fmaf(v.m, c.scale, kLn2 * log2_s);
    if (c.entropy) c.entropy[row] = empty ? 0.f : kLn2 * (log2_s - v.t / v.s);
    if (c.logprobs) c.logprobs[row] = token >= 0 && token < c.vocab ? logprob(logit) : 0.f;      // (a row that is not scored gets 0)
  }
  if (TOP && (int)threadIdx.x < c.top) {
    const uint64_t key = best[threadIdx.x];
    c.top_ids[(int64_t)row * c.top + threadIdx.x] = index_of(key);
    c.top_logprobs[(int64_t)row * c.top + threadIdx.x] = logprob(value_of((uint32_t)(key >> 32)));
  }
}

template <typename T, bool TOP, int PIECES, bool STREAM>
__global__ __launch_bounds__(kThreads) void rows_kernel(LogprobCall c) {
  constexpr int kChunk = kThreads * PIECES * 8;
  __shared__ Stats parts[kThreads / 64];
  __shared__ std::conditional_t<TOP, TopLds, char> lds;
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const int begin = (int)((int64_t)c.chunks * split / c.splits), end = (int)((int64_t)c.chunks * (split + 1) / c.splits);
  const T* logits = static_cast<const T*>(c.logits) + row * c.stride;
  const float scale2 = c.scale * kLog2e;
  Stats v = {-INFINITY, 0.f, 0.f};
  float bound = -INFINITY;
  int n_list = 0;
  if constexpr (TOP) clear_list(lds);
  const bool asked = c.splits == 1 && c.logprobs && threadIdx.x == 0;
  const int token = asked ? c.tokens[row] : -1;
  for (int chunk = begin; chunk < end; ++chunk) {
    const int first = chunk * kChunk;
    const int last = c.vocab;
    Piece<T> x[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int col = first + (p * kThreads + (int)threadIdx.x) * 8;
      if (col + 8 <= last) {
        x[p] = piece_at<STREAM>(logits + col);
      } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = col + i < last ? one_value(logits[col + i]) : -INFINITY;
        narrow(f, x[p]);
      }
    }
    float most = -INFINITY;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, value_at(x[p], i));
    const float m = fmaxf(v.m, most);
    const float base = m == -INFINITY ? 0.f : m;                // (all masked so far: exponents of -inf, not NaN)
    if (v.m != -INFINITY) {
      const float d = (v.m - base) * scale2, w = __builtin_amdgcn_exp2f(d);
      v.t = (v.t + v.s * fmaxf(d, kLow)) * w;
      v.s *= w;
    }
    v.m = m;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = (value_at(x[p], i) - base) * scale2;
        const float e = __builtin_amdgcn_exp2f(d);
        v.s += e;
        v.t = __builtin_fmaf(e, fmaxf(d, kLow), v.t);
      }
    if constexpr (TOP) top_of_chunk<T, PIECES>(lds, x, logits, first, last, c.top, most, v.s != v.s, bound, n_list);
  }
  const float logit = logit_of<T>(c, row, token);
  const uint64_t* best = nullptr;
  if constexpr (TOP) {
    rank_list(lds, n_list, c.top);
    best = lds.best;
  }
  v = stats_of_block(v, parts, scale2);
  if (c.splits == 1) {
    finish_row<TOP>(c, row, v, best, token, logit);
  } else {
    const int64_t at = (int64_t)row * c.splits + split;
    if (threadIdx.x == 0) *part_stats(c, at) = v;
    if (TOP && (int)threadIdx.x < c.top) part_best(c, at)[threadIdx.x] = best[threadIdx.x];
  }
}

// A row's parts: a lane each, joined over lanes; of their lists, what reaches a bound that k entries reach is ranked.
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void join_kernel(LogprobCall c) {
  __shared__ std::conditional_t<TOP, TopLds, char> lds;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int64_t at = (int64_t)row * c.splits;
  // Everything that is read is asked for at once (keys: a batch of them).
  constexpr int kEach = 3, kBatch = kEach * kThreads;
  static_assert(kBatch + kMostTop <= kList, "a batch and the best before it");
  const int n = c.splits * c.top, k = c.top;
  const uint64_t* lists = part_best(c, at);
  const int token = c.logprobs && threadIdx.x == 0 ? c.tokens[row] : -1;
  Stats v = {-INFINITY, 0.f, 0.f};
  if (lane < c.splits) v = *part_stats(c, at + lane);
  uint64_t keys[kEach] = {};
  // Entry `deep` of every list and those before it are k at least: k entries reach the least of these; or, with as many lists as k, the
  // k-th largest of their first.
  const int deep = (k + c.splits - 1) / c.splits - 1;
  uint32_t head = 0;
  if constexpr (TOP) {
    if (lane < c.splits) head = (uint32_t)(lists[lane * k + deep] >> 32);
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (e * kThreads + (int)threadIdx.x < n) keys[e] = lists[e * kThreads + threadIdx.x];
    clear_list(lds);
  }
  const float logit = logit_of<T>(c, row, token);
  v = stats_of_wave(v, c.scale * kLog2e);
  const uint64_t* best = nullptr;
  if constexpr (TOP) {
    uint32_t bound;
    if (deep == 0) {
      const uint32_t upper[1] = {head >> 16};
      bound = kth_of_wave(upper, k) << 16;
    } else {
      bound = lane < c.splits ? head : 0xffffffffu;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) bound = min(bound, (uint32_t)__shfl_xor(bound, m));
    }
    __syncthreads();
    for (int first = 0;;) {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (keys[e] != 0 && (uint32_t)(keys[e] >> 32) >= bound) lds.list[atomicAdd(&lds.n, 1)] = keys[e];
      __syncthreads();
      rank_list(lds, lds.n, k);
      first += kBatch;
      if (first >= n) break;
      restart_list(lds, k);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = first + e * kThreads + (int)threadIdx.x;
        keys[e] = i < n ? lists[i] : 0;
      }
    }
    best = lds.best;
  }
  finish_row<TOP>(c, row, v, best, token, logit);
}

// Pieces of a thread a turn.  fp32 loads of all of them are in flight together; bf16 ones, which load_piece widens behind each load, one at a time.
constexpr int kGradPieces = 4;
template <typename T>
__global__ __launch_bounds__(kThreads) void grad_kernel(LogprobGradCall c) {
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const T* logits = static_cast<const T*>(c.logits) + row * c.stride;
  T* out = static_cast<T*>(c.out) + row * c.out_stride;
  const float lse = c.lse[row];
  // A row of nothing but masked logits, by -inf or by a value so low that lse, in 32 bits, is that value: all its gradients are 0.
  const bool empty = lse < kMaskedLse;
  // (subtracted before the change of base: both sides times log2(e) would each be rounded at the logits' size, not at their distance's)
  const float from = empty ? 0.f : lse;
  const int token = c.tokens && !empty ? c.tokens[row] : -1;
  const bool asked = token >= 0 && token < c.vocab;
  const float g = c.grad_logprobs && asked ? c.grad_logprobs[row] * c.scale : 0.f;
  const float gh = c.grad_entropy ? c.grad_entropy[row] * c.scale : 0.f;
  const float entropy = c.grad_entropy ? c.entropy[row] : 0.f;
  // -p (g + gh (lp + H)) with lp in base 2
  const float a = -(g + gh * entropy), b = -gh * kLn2;
  const int pieces = (c.vocab + 7) / 8;
  const int first = (int)((int64_t)pieces * split / c.splits), end = (int)((int64_t)pieces * (split + 1) / c.splits);
  for (int p0 = first + threadIdx.x; p0 < end; p0 += kThreads * kGradPieces) {
    float x[kGradPieces][8];
#pragma unroll
    for (int u = 0; u < kGradPieces; ++u)
      if (p0 + u * kThreads < end) load_piece(logits, (p0 + u * kThreads) * 8, c.vocab, x[u]);
#pragma unroll
    for (int u = 0; u < kGradPieces; ++u) {
      const int col = (p0 + u * kThreads) * 8;
      if (p0 + u * kThreads >= end) break;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = __builtin_fmaf(x[u][i], c.scale, -from) * kLog2e;
        const float w = __builtin_amdgcn_exp2f(d);
        x[u][i] = w * __builtin_fmaf(b, fmaxf(d, kLow), a);
      }
      if (asked && (unsigned)(token - col) < 8u) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (token - col == i) x[u][i] += g;
      }
      store_piece(out, col, c.vocab, x[u]);
    }
  }
}

}  // namespace

// Chunks of a row and workgroups it is split over.  Many rows fill the card by themselves, and rows of two chunks are not worth the launch
// that joins them (64 x 32000 fp32: 4.7 + 3.2 us split, 5.7 whole; with the 20 most likely tokens 11.3 in all split, 11.5 whole, but
// 4 x 32000 8.8 and 10.5); few rows are spread over workgroups, as many as fill the compute units twice, in chunks of a quarter of the
// size where those of the full size do not fill them once.  (512 x 131072 bf16, 20 most likely: 48 us whole, 59 in two.)
static int chunks_of(int vocab, int pieces) { return (int)(((int64_t)vocab + kThreads * 8 * pieces - 1) / (kThreads * 8 * pieces)); }
static bool whole_rows(int rows, int vocab, int top) { return rows >= 512 || chunks_of(vocab, kPieces) <= (top > 0 && rows < 64 ? 1 : 2); }
static bool small_chunks(int rows, int vocab, int top) { return !whole_rows(rows, vocab, top) && (int64_t)rows * chunks_of(vocab, kPieces) < 256; }
static int logprob_chunks(int rows, int vocab, int top) { return chunks_of(vocab, small_chunks(rows, vocab, top) ? kFewPieces : kPieces); }
static int logprob_splits(int rows, int vocab, int top) {
  if (whole_rows(rows, vocab, top)) return 1;
  const int chunks = logprob_chunks(rows, vocab, top), want = (512 + rows - 1) / rows;
  const int most = want < kMostSplits ? want : kMostSplits;
  return most < chunks ? most : chunks;
}
size_t logprob_workspace(int rows, int vocab, int top) {
  const int splits = logprob_splits(rows, vocab, top);
  if (splits <= 1) return 0;
  const size_t parts = (size_t)rows * splits;
  return (parts * sizeof(Stats) + 7) / 8 * 8 + parts * top * sizeof(uint64_t);
}

// More logits than a cache holds are read with non-temporal loads (us, plain / non-temporal: 4096 x 128011 bf16 189 / 164, 2048 rows 97 / 87); not
// with the most likely tokens, whose ranking bounds them (20 of them, 512 x 131072 bf16 47.6 / 47.0, 256 x 131072 fp32 38.4 / 40.0).
template <typename T, bool TOP>
static hipError_t launch_rows(const LogprobCall& c, hipStream_t stream) {
  const dim3 grid((unsigned)c.rows * c.splits), block(kThreads);
  if (small_chunks(c.rows, c.vocab, c.top)) hipLaunchKernelGGL((rows_kernel<T, TOP, kFewPieces, false>), grid, block, 0, stream, c);
  else if (!TOP && c.rows * (int64_t)c.vocab * (int64_t)sizeof(T) > kStreamBytes) hipLaunchKernelGGL((rows_kernel<T, TOP, kPieces, !TOP>), grid, block, 0, stream, c);
  else hipLaunchKernelGGL((rows_kernel<T, TOP, kPieces, false>), grid, block, 0, stream, c);
  if (hipError_t e = hipGetLastError()) return e;
  if (c.splits > 1) hipLaunchKernelGGL((join_kernel<T, TOP>), dim3((unsigned)c.rows), block, 0, stream, c);
  return hipGetLastError();
}

hipError_t launch_logprobs(LogprobCall c, int dtype, hipStream_t stream) {
  c.chunks = logprob_chunks(c.rows, c.vocab, c.top);
  c.splits = logprob_splits(c.rows, c.vocab, c.top);
  if (dtype == RLKV_F32) return c.top ? launch_rows<float, true>(c, stream) : launch_rows<float, false>(c, stream);
  return c.top ? launch_rows<uint16_t, true>(c, stream) : launch_rows<uint16_t, false>(c, stream);
}

hipError_t launch_logprobs_grad(LogprobGradCall c, int dtype, hipStream_t stream) {
  const int pieces = (c.vocab + 7) / 8;
  const int most = (pieces + kThreads * 4 - 1) / (kThreads * 4), want = (4096 + c.rows - 1) / c.rows;
  c.splits = want < most ? want : most;
  if (c.splits < 1) c.splits = 1;
  if (dtype == RLKV_F32) hipLaunchKernelGGL(grad_kernel<float>, dim3((unsigned)c.rows * c.splits), dim3(kThreads), 0, stream, c);
  else hipLaunchKernelGGL(grad_kernel<uint16_t>, dim3((unsigned)c.rows * c.splits), dim3(kThreads), 0, stream, c);
  return hipGetLastError();
}

}  // namespace rlkv
