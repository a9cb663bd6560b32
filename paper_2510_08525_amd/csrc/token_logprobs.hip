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
// it holds in registers.  The k-th largest of the 64 lanes' maxima of a wavefront is a value that at least k logits of the chunk
// reach; the largest such bound of the workgroup, or the k-th best so far where that is more, lets few logits through, which are collected in LDS and
// ranked by counting.  A chunk that lets through more than the list holds (ties, masks) is searched maximum by maximum.
// Few rows are split over workgroups, whose partial results a second kernel joins in a fixed order.
// Bound: HBM; 6 or 7 vector instructions and an exponential a logit are not far behind.
#include <type_traits>

#include "token_ops.h"

namespace rlkv {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256;
constexpr int kPieces = 8;                              // pieces of eight logits of a thread in a chunk
constexpr int kChunk = kThreads * kPieces * 8;
constexpr int kList = 1024;                             // candidates a workgroup ranks at once
constexpr float kMaskedLse = -1e30f;
constexpr float kLow = -256.f;                          // in the place of exponents so low that their weight is 0

struct Stats { float m, s, t; };                        // maximum of the logits, sum, weighted sum (exponents of base 2)

__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float scale2) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return Stats{m, a.s + b.s, a.t + b.t};      // (sums of zeros; a NaN stays one)
  const float da = (a.m - m) * scale2, db = (b.m - m) * scale2;
  const float wa = __builtin_amdgcn_exp2f(da), wb = __builtin_amdgcn_exp2f(db);
  return Stats{m, a.s * wa + b.s * wb, (a.t + a.s * fmaxf(da, kLow)) * wa + (b.t + b.s * fmaxf(db, kLow)) * wb};
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
// The k-th largest (k from 1) of the 64 lanes' values: how many are larger, and how many equal ones have a lower lane.
__device__ __forceinline__ uint32_t kth_of_wave(uint32_t x, int k) {
  const int lane = threadIdx.x & 63;
  int rank = 0;
  for (int i = 0; i < 64; ++i) {
    const uint32_t y = __builtin_amdgcn_readlane(x, i);
    rank += y > x || (y == x && i < lane);
  }
  const uint64_t at = __ballot(rank == k - 1);
  return __builtin_amdgcn_readlane(x, __builtin_ctzll(at));
}

struct TopLds {
  uint64_t best[kMostTop];          // the best so far, largest first, 0 = none
  uint64_t list[kList];
  uint64_t wave_best[kThreads / 64];
  uint32_t bound[kThreads / 64];
  int32_t n;
};

// list[0, n) (distinct keys, n <= kList, all threads past a barrier) -> the k largest of them into best, in order.
__device__ void rank_list(TopLds& lds, int n, int k) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t x = lds.list[i];
    int rank = 0;
    for (int o = 0; o < n; ++o) rank += lds.list[o] > x;
    if (rank < k) lds.best[rank] = x;
  }
  if ((int)threadIdx.x >= n && (int)threadIdx.x < k) lds.best[threadIdx.x] = 0;
  __syncthreads();
}

// Brings the chunk that starts at column `first` (valid: below `last`), in x, into the best k.
__device__ void top_of_chunk(TopLds& lds, const float (&x)[kPieces][8], int first, int last, int k) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  uint32_t most = 0;
#pragma unroll
  for (int p = 0; p < kPieces; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = first + (p * kThreads + tid) * 8 + i;
      const uint32_t o = col < last ? order_of(x[p][i]) : 0;
      most = o > most ? o : most;
    }
  const uint32_t own = kth_of_wave(most, k);
  if (lane == 0) lds.bound[wave] = own;
  if (tid < k) lds.list[tid] = lds.best[tid];
  if (tid == 0) lds.n = k;
  __syncthreads();
  uint64_t bound = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) bound = lds.bound[w] > bound ? lds.bound[w] : bound;
  bound <<= 32;                                                  // (equal values pass, whatever their index)
  const uint64_t worst = lds.best[k - 1];
  bound = worst > bound ? worst : bound;
  bool any = (uint64_t)most << 32 >= (bound & 0xffffffff00000000ull);
  if (any) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = first + (p * kThreads + tid) * 8 + i;
        if (col >= last) continue;
        const uint64_t key = key_of(x[p][i], col);
        if (key < bound) continue;
        const int at = atomicAdd(&lds.n, 1);
        if (at < kList) lds.list[at] = key;
      }
  }
  __syncthreads();
  const int n = lds.n;
  __syncthreads();
  if (n <= kList) {
    // (places that hold no key yet are 0 and equal: they rank behind all keys, where nothing reads more than a 0)
    rank_list(lds, n, k);
    return;
  }
  // Maximum by maximum, each below the one before; list[0, k) still has the best of the chunks before.
  uint64_t below = ~0ull;
  for (int r = 0; r < k; ++r) {
    uint64_t best = tid < k && lds.list[tid] < below ? lds.list[tid] : 0;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int col = first + (p * kThreads + tid) * 8 + i;
        if (col >= last) continue;
        const uint64_t key = key_of(x[p][i], col);
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

__device__ __forceinline__ Stats stats_of_block(Stats v, Stats (&parts)[kThreads / 64], float scale2) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = join(v, Stats{__shfl_xor(v.m, m), __shfl_xor(v.s, m), __shfl_xor(v.t, m)}, scale2);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
  __syncthreads();
  v = parts[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v = join(v, parts[w], scale2);
  return v;
}

// What a row's results are made of: in the workspace, per row and split.
__device__ __forceinline__ Stats* part_stats(const LogprobCall& c, int64_t at) { return static_cast<Stats*>(c.workspace) + at; }
__device__ __forceinline__ uint64_t* part_best(const LogprobCall& c, int64_t at) {
  const size_t stats = ((size_t)c.rows * c.splits * sizeof(Stats) + 7) / 8 * 8;
  return reinterpret_cast<uint64_t*>(static_cast<char*>(c.workspace) + stats) + at * c.top;
}

template <typename T, bool TOP>
__device__ void finish_row(const LogprobCall& c, int row, const Stats& v, const uint64_t* best) {
  const float scale2 = c.scale * kLog2e, log2_s = log2f(v.s);
  const bool empty = v.s == 0.f;                                // (nothing but masked logits)
  auto logprob = [&](float x) { return empty ? -INFINITY : kLn2 * ((x - v.m) * scale2 - log2_s); };
  if (threadIdx.x == 0) {
    if (c.lse) c.lse[row] = empty ? -INFINITY : __builtin_fmaf(v.m, c.scale, kLn2 * log2_s);
    if (c.entropy) c.entropy[row] = empty ? 0.f : kLn2 * (log2_s - v.t / v.s);
    if (c.logprobs) {
      const int token = c.tokens[row];
      const bool asked = token >= 0 && token < c.vocab;         // (a row that is not scored gets 0)
      c.logprobs[row] = asked ? logprob(one_value((static_cast<const T*>(c.logits) + row * c.stride)[token])) : 0.f;
    }
  }
  if (TOP && (int)threadIdx.x < c.top) {
    const uint64_t key = best[threadIdx.x];
    c.top_ids[(int64_t)row * c.top + threadIdx.x] = index_of(key);
    c.top_logprobs[(int64_t)row * c.top + threadIdx.x] = logprob(value_of((uint32_t)(key >> 32)));
  }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void rows_kernel(LogprobCall c) {
  __shared__ Stats parts[kThreads / 64];
  __shared__ std::conditional_t<TOP, TopLds, char> lds;
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const int begin = (int)((int64_t)c.chunks * split / c.splits), end = (int)((int64_t)c.chunks * (split + 1) / c.splits);
  const T* logits = static_cast<const T*>(c.logits) + row * c.stride;
  const float scale2 = c.scale * kLog2e;
  Stats v = {-INFINITY, 0.f, 0.f};
  if constexpr (TOP) {
    if ((int)threadIdx.x < c.top) lds.best[threadIdx.x] = 0;
    __syncthreads();
  }
  for (int chunk = begin; chunk < end; ++chunk) {
    const int first = chunk * kChunk;
    const int last = c.vocab;
    float x[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int col = first + (p * kThreads + (int)threadIdx.x) * 8;
      if (col + 8 <= last) {
        widen(*reinterpret_cast<const Piece<T>*>(logits + col), x[p]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[p][i] = col + i < last ? one_value(logits[col + i]) : -INFINITY;
      }
    }
    float m = v.m;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, x[p][i]);
    const float base = m == -INFINITY ? 0.f : m;                // (all masked so far: exponents of -inf, not NaN)
    if (v.m != -INFINITY) {
      const float d = (v.m - base) * scale2, w = __builtin_amdgcn_exp2f(d);
      v.t = (v.t + v.s * fmaxf(d, kLow)) * w;
      v.s *= w;
    }
    v.m = m;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = (x[p][i] - base) * scale2;
        const float e = __builtin_amdgcn_exp2f(d);
        v.s += e;
        v.t = __builtin_fmaf(e, fmaxf(d, kLow), v.t);
      }
    if constexpr (TOP) top_of_chunk(lds, x, first, last, c.top);
  }
  v = stats_of_block(v, parts, scale2);
  const uint64_t* best = nullptr;
  if constexpr (TOP) best = lds.best;
  if (c.splits == 1) {
    finish_row<T, TOP>(c, row, v, best);
  } else {
    const int64_t at = (int64_t)row * c.splits + split;
    if (threadIdx.x == 0) *part_stats(c, at) = v;
    if (TOP && (int)threadIdx.x < c.top) part_best(c, at)[threadIdx.x] = best[threadIdx.x];
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(LogprobCall c) {
  __shared__ TopLds lds;
  const int row = blockIdx.x;
  const int64_t at = (int64_t)row * c.splits;
  Stats v = *part_stats(c, at);
  for (int s = 1; s < c.splits; ++s) v = join(v, *part_stats(c, at + s), c.scale * kLog2e);
  if (c.top) {
    if ((int)threadIdx.x < c.top) lds.best[threadIdx.x] = 0;
    __syncthreads();
    const int n = c.splits * c.top;
    for (int first = 0; first < n; first += kList - kMostTop) {
      const int some = n - first < kList - kMostTop ? n - first : kList - kMostTop;
      for (int i = threadIdx.x; i < some; i += kThreads) lds.list[c.top + i] = part_best(c, at)[first + i];
      if ((int)threadIdx.x < c.top) lds.list[threadIdx.x] = lds.best[threadIdx.x];
      __syncthreads();
      rank_list(lds, c.top + some, c.top);
    }
  }
  finish_row<T, true>(c, row, v, lds.best);
}

constexpr int kGradPieces = 4;                          // pieces of a thread whose loads are in flight together
template <typename T>
__global__ __launch_bounds__(kThreads) void grad_kernel(LogprobGradCall c) {
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const T* logits = static_cast<const T*>(c.logits) + row * c.stride;
  T* out = static_cast<T*>(c.out) + row * c.out_stride;
  const float scale2 = c.scale * kLog2e;
  const float lse = c.lse[row];
  // A row of nothing but masked logits, by -inf or by a value so low that lse, in 32 bits, is that value: all its gradients are 0.
  const bool empty = lse < kMaskedLse;
  const float lse2 = empty ? 0.f : lse * kLog2e;
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
        const float d = __builtin_fmaf(x[u][i], scale2, -lse2);
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

int logprob_chunks(int vocab) { return (vocab + kChunk - 1) / kChunk; }

// Workgroups a row is split over: as many as fill the card some times over, one per chunk at most.
int logprob_splits(int rows, int vocab) {
  const int chunks = logprob_chunks(vocab);
  if (rows >= 1024) return 1;
  const int want = (1024 + rows - 1) / rows;
  return want < chunks ? want : chunks;
}
size_t logprob_workspace(int rows, int vocab, int top) {
  const size_t parts = (size_t)rows * logprob_splits(rows, vocab);
  if (logprob_splits(rows, vocab) <= 1) return 0;
  return (parts * sizeof(Stats) + 7) / 8 * 8 + parts * top * sizeof(uint64_t);
}

hipError_t launch_logprobs(LogprobCall c, int dtype, hipStream_t stream) {
  c.chunks = logprob_chunks(c.vocab);
  c.splits = logprob_splits(c.rows, c.vocab);
  auto run = [&](auto rows, auto join) {
    hipLaunchKernelGGL(rows, dim3((unsigned)c.rows * c.splits), dim3(kThreads), 0, stream, c);
    if (hipError_t e = hipGetLastError()) return e;
    if (c.splits > 1) hipLaunchKernelGGL(join, dim3((unsigned)c.rows), dim3(kThreads), 0, stream, c);
    return hipGetLastError();
  };
  if (dtype == RLKV_F32) return c.top ? run(rows_kernel<float, true>, join_kernel<float>) : run(rows_kernel<float, false>, join_kernel<float>);
  return c.top ? run(rows_kernel<uint16_t, true>, join_kernel<uint16_t>) : run(rows_kernel<uint16_t, false>, join_kernel<uint16_t>);
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
