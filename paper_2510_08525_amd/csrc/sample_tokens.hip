// A token of every row of logits, drawn by a given random number:
//
//   w[i] = exp((x[i] - max x) / temperature);  in order of x (equal ones by the lower token) the first top_k are kept, of those the first whose
//   weights reach top_p of their sum, of those the ones with w >= min_p;  token = first kept i with  sum of kept w[0 .. i] > u * sum of kept w
//
// Weights are whole numbers of 2^-bits, bits = 62 - log2(vocab), from an exponential in 64 bits: their sums are exact in 64-bit integers, in whatever
// order they are formed, so atomics and scans give the same token at every call, and borders between tokens are within 2^-bits of where the
// formula has them (2^-45 for 131072 tokens; what fp32 sums leave, 2^-24 of a border's place, changes a token of 128k in one of hundred rows).
#include "sample_tokens.h"
#include "token_ops.h"

namespace rlkv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
constexpr int kTileTokens = kThreads * 8;
constexpr float kBinsPerUnit = 32.f;      // bins of the first turn: the way from the largest logit over the temperature, 64 of it

// Ascending with x; zeros of either sign are the same.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Smem {
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  unsigned long long sums[kWaves];
  uint32_t low[kWaves], high[kWaves];
  unsigned long long found_before, found_mass;
  uint32_t found, found_count;
  int32_t index;
};

__device__ __forceinline__ unsigned long long sum_over_wave(unsigned long long x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

struct Row {
  double top, inv_t;        // largest logit, 1 / temperature
  double unit;              // weight 1 in whole numbers
  double least;             // the logit's way from the largest over the temperature below which a weight is 0
  double min_w;             // least weight that is kept
  // a token is kept if its key is above `key`, or is `key` and its place is at most `last`
  uint32_t key;
  int32_t last;
};
__device__ __forceinline__ unsigned long long weight_of(const Row& r, float x) {
  const double z = ((double)x - r.top) * r.inv_t;
  if (!(z >= r.least)) return 0;           // (a masked logit's place is -infinity, or NaN where the temperature is infinite)
  const double w = exp(z);
  return w >= r.min_w ? (unsigned long long)(w * r.unit + 0.5) : 0;
}
__device__ __forceinline__ bool keeps(const Row& r, float x, int i) {
  const uint32_t key = key_of(x);
  return key > r.key || (key == r.key && i <= r.last);
}

// f(x, i) for the tokens [lo, hi) of the row, in pieces of eight, `threads` of them side by side of which this is number t.
template <typename T, typename F>
__device__ __forceinline__ void each_token(const T* row, int lo, int hi, int t, int threads, F f) {
  for (int64_t at = lo + (int64_t)t * 8; at < hi; at += (int64_t)threads * 8) {
    float x[8];
    load_piece(row, (int)at, hi, x);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < hi) f(x[i], (int)at + i);
  }
}

// First place in [lo, hi) where the running sum of f is above `target`, in all threads.  The sum over [lo, hi) has to be.
template <typename T, typename F>
__device__ int place_of(Smem& sm, const T* row, int lo, int hi, unsigned long long target, F f) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  while (hi - lo > kTileTokens) {            // sixteen parts, one a wavefront
    const int part = ((hi - lo + kWaves - 1) / kWaves + 7) / 8 * 8;
    const int64_t a = lo + (int64_t)wave * part, b = a + part;
    unsigned long long sum = 0;
    if (a < hi) each_token(row, (int)a, (int)(b < hi ? b : hi), lane, 64, [&](float x, int i) { sum += f(x, i); });
    sum = sum_over_wave(sum);
    __syncthreads();
    if (lane == 0) sm.sums[wave] = sum;
    __syncthreads();
    int w = 0;
    for (; w < kWaves - 1 && target >= sm.sums[w]; ++w) target -= sm.sums[w];
    lo += w * part;
    hi = lo + part < hi ? lo + part : hi;
  }
  // eight tokens a thread
  float x[8];
  const int at = lo + threadIdx.x * 8;
  unsigned long long v[8], sum = 0;
  if (at < hi) load_piece(row, at, hi, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = at + i < hi ? f(x[i], at + i) : 0;
    sum += v[i];
  }
  unsigned long long before = sum;           // inclusive over the wavefront's lanes
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long y = __shfl_up(before, d);
    if (lane >= d) before += y;
  }
  __syncthreads();
  if (lane == 63) sm.sums[wave] = before;
  __syncthreads();
  before -= sum;
  for (int w = 0; w < wave; ++w) before += sm.sums[w];
  if (before <= target && target < before + sum) {
    int i = 0;
    unsigned long long run = before;
    for (; i < 7 && run + v[i] <= target; ++i) run += v[i];
    sm.index = at + i;
  }
  __syncthreads();
  return sm.index;
}

// The bin in which the running sum (of counts, or of masses) passes `target`; found_before: the sum in front of it.
__device__ void bin_of(Smem& sm, bool by_mass, unsigned long long target) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, b = threadIdx.x * 2;
  const unsigned long long x = by_mass ? sm.mass[b] : sm.count[b], y = by_mass ? sm.mass[b + 1] : sm.count[b + 1];
  unsigned long long run = x + y;
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long other = __shfl_up(run, d);
    if (lane >= d) run += other;
  }
  if (lane == 63) sm.sums[wave] = run;
  __syncthreads();
  run -= x + y;
  for (int w = 0; w < wave; ++w) run += sm.sums[w];
  if (run <= target && target < run + x + y) {
    const bool second = target >= run + x;
    sm.found = b + second;
    sm.found_before = run + (second ? x : 0);
    sm.found_mass = sm.mass[b + second];
    sm.found_count = sm.count[b + second];
  }
  __syncthreads();
}

// Cuts the kept tokens of `r` to the first ones in order of their logits: to `target` of them, or (by_mass) to those in front of which the weights
// sum to less than `target`.  There are more of them.
template <typename T>
__device__ void cut(Smem& sm, const T* row, int vocab, Row& r, bool by_mass, unsigned long long target) {
  const float top = (float)r.top, per = (float)r.inv_t * kBinsPerUnit;
  auto first_bin = [&](float x) {
    const float z = (top - x) * per;
    return z < (float)(kBins - 1) ? (int)z : kBins - 1;       // (NaN, of a masked logit at an infinite temperature: the last)
  };
  auto add = [&](int bin, float x) {
    atomicAdd(&sm.count[bin], 1u);
    if (by_mass) {
      const unsigned long long w = weight_of(r, x);
      if (w) atomicAdd(&sm.mass[bin], w);
    }
  };
  auto clear = [&]() {
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      sm.mass[b] = 0;
      sm.count[b] = 0;
    }
    __syncthreads();
  };
  const unsigned long long last = target - 1;      // (the token that reaches the target is kept)
  clear();
  each_token(row, 0, vocab, threadIdx.x, kThreads, [&](float x, int i) {
    if (keeps(r, x, i)) add(first_bin(x), x);
  });
  __syncthreads();
  bin_of(sm, by_mass, last);
  const int bin = sm.found;
  unsigned long long before = sm.found_before;
  // the keys of that bin, and by them bins of fewer and fewer keys
  uint32_t low = 0xffffffffu, high = 0;
  each_token(row, 0, vocab, threadIdx.x, kThreads, [&](float x, int i) {
    if (first_bin(x) != bin || !keeps(r, x, i)) return;
    const uint32_t k = key_of(x);
    low = k < low ? k : low;
    high = k > high ? k : high;
  });
  for (int d = 32; d; d >>= 1) {
    low = min(low, (uint32_t)__shfl_xor(low, d));
    high = max(high, (uint32_t)__shfl_xor(high, d));
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    sm.low[threadIdx.x >> 6] = low;
    sm.high[threadIdx.x >> 6] = high;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    low = min(low, sm.low[w]);
    high = max(high, sm.high[w]);
  }
  for (;;) {
    const int bits = 32 - __clz(high - low);           // (0 for one key)
    const int shift = bits > 11 ? bits - 11 : 0;
    clear();
    each_token(row, 0, vocab, threadIdx.x, kThreads, [&](float x, int i) {
      const uint32_t k = key_of(x);
      if (k >= low && k <= high && keeps(r, x, i)) add((int)((high - k) >> shift), x);
    });
    __syncthreads();
    bin_of(sm, by_mass, last - before);
    before += sm.found_before;
    const uint32_t at = high - (sm.found << shift), to = at - ((1u << shift) - 1);
    low = to > at || to < low ? low : to;
    high = at;
    if (shift == 0) break;
  }
  // one key: of its tokens those that are needed, by their places
  const uint32_t count = sm.found_count;
  unsigned long long need = last - before + 1;
  if (by_mass) {
    const unsigned long long each = sm.found_mass / count;      // (equal logits have equal weights, none of them 0 here)
    need = (need + each - 1) / each;
  }
  __syncthreads();
  const int32_t old_last = high == r.key ? r.last : 0x7fffffff;
  int32_t place = old_last;
  if (need < count) place = place_of(sm, row, 0, vocab, need - 1, [&](float x, int i) { return (unsigned long long)(key_of(x) == high && i <= old_last); });
  r.key = high;
  r.last = place;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleCall c, int bits) {
  __shared__ Smem sm;
  const int64_t n = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  const double t = c.temperatures ? c.temperatures[n] : c.temperature;
  const double top_p = c.top_ps ? c.top_ps[n] : c.top_p, min_p = c.min_ps ? c.min_ps[n] : c.min_p;
  const int top_k = c.top_ks ? c.top_ks[n] : c.top_k;
  float top = -INFINITY;
  bool bad = false;
  each_token(row, 0, c.vocab, threadIdx.x, kThreads, [&](float x, int) {
    top = fmaxf(top, x);
    bad |= !(x < INFINITY);
  });
  top = max_of_wave(top);
  if (lane == 0) sm.sums[wave] = __float_as_uint(top);
  bad = __syncthreads_or(bad);
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, __uint_as_float((uint32_t)sm.sums[w]));
  __syncthreads();
  if (bad || top == -INFINITY) {             // nothing to draw from
    if (threadIdx.x == 0) {
      c.tokens[n] = -1;
      if (c.logprobs) c.logprobs[n] = NAN;
    }
    return;
  }
  if (!(t > 0.)) {
    const int i = place_of(sm, row, 0, c.vocab, 0, [&](float x, int) { return (unsigned long long)(x == top); });
    if (threadIdx.x == 0) {
      c.tokens[n] = i;
      if (c.logprobs) c.logprobs[n] = 0.f;
    }
    return;
  }
  Row r;
  r.top = top;
  r.inv_t = 1. / t;
  r.unit = (double)(1ull << bits);
  r.least = -(bits + 1) * 0.69314718055994530942;
  r.min_w = 0.;
  r.key = 0;
  r.last = 0x7fffffff;
  auto kept_weight = [&](float x, int i) { return keeps(r, x, i) ? weight_of(r, x) : 0ull; };
  auto total_of = [&]() {
    unsigned long long sum = 0;
    each_token(row, 0, c.vocab, threadIdx.x, kThreads, [&](float x, int i) { sum += kept_weight(x, i); });
    sum = sum_over_wave(sum);
    __syncthreads();
    if (lane == 0) sm.sums[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kWaves; ++w) sum += sm.sums[w];
    __syncthreads();
    return sum;
  };
  if (top_k > 0 && top_k < c.vocab) cut(sm, row, c.vocab, r, false, top_k);
  if (top_p < 1.) {
    const unsigned long long total = total_of();
    // sums in front of a kept token are below p * total: whole numbers below its ceiling; the first token is kept always
    const double p = top_p > 0. ? top_p : 0.;
    const unsigned long long p64 = (unsigned long long)(p * 18446744073709551616.);
    const unsigned long long target = __umul64hi(total, p64) + (total * p64 != 0);
    cut(sm, row, c.vocab, r, true, target > 0 ? target : 1);
  }
  r.min_w = min_p > 0. ? (min_p < 1. ? min_p : 1.) : 0.;
  const unsigned long long total = total_of();
  const float u = c.uniforms[n];
  const unsigned long long u64 = !(u > 0.f) ? 0 : u < 1.f ? (unsigned long long)((double)u * 18446744073709551616.) : ~0ull;
  const int i = place_of(sm, row, 0, c.vocab, __umul64hi(total, u64), kept_weight);
  if (threadIdx.x == 0) {
    c.tokens[n] = i;
    if (c.logprobs) c.logprobs[n] = (float)(((double)one_value(row[i]) - r.top) * r.inv_t - log((double)total / r.unit));
  }
}

}  // namespace

size_t sample_workspace(int, int) { return 0; }

hipError_t launch_sample(const SampleCall& c, int dtype, hipStream_t stream) {
  int bits = 62;
  for (int64_t n = 1; n < c.vocab; n *= 2) --bits;
  if (dtype == RLKV_F32) sample_kernel<float><<<(unsigned)c.rows, kThreads, 0, stream>>>(c, bits);
  else sample_kernel<uint16_t><<<(unsigned)c.rows, kThreads, 0, stream>>>(c, bits);
  return hipGetLastError();
}

}  // namespace rlkv
