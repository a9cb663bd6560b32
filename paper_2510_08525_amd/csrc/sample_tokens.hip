// A token of every row of logits, drawn by a given random number:
//
//   w[i] = exp((x[i] - max x) / temperature);  in order of x (equal ones by the lower token) the first top_k are kept, of those the first whose
//   weights reach top_p of their sum, of those the ones with w >= min_p;  token = first kept i with  sum of kept w[0 .. i] > u * sum of kept w
//
// Weights are whole numbers of 2^-bits, bits = min(50, 62 - log2(vocab)), from an exponential in 64 bits: their sums are exact in 64-bit integers, in
// whatever order they are formed, so atomics and scans give the same token at every call, and borders between tokens are where the formula has
// them to 2^-38 of the weights (what sums in 32 bits leave, 2^-24 of a border's place, changes a token of 128k in one of hundred rows).
//
// A row is read by as many workgroups as it has parts of 8192 tokens.  Launches, of which rows without filters need the first and the last:
//   parts    largest logit and, for rows whose sum is asked for, the sum of weights of a part
//   bins     how many tokens, and what weight, lie in each of 4096 steps down from the largest logit
//   collect  the step in which the cut falls: its tokens go into a list; the weight of a part's tokens above it
//   draw     one workgroup a row: the cut among the list's tokens, the part that the number falls into, the token in it
// Of rows with top_k the two in the middle do nothing where a logit that top_k tokens reach is found among the largest ones of each 128 tokens: the
// last launch makes the list, from the chunks that reach it, and finds the token in the list (48 rows of 128011 in float32, most with a
// top_k: 38 to 45 us, with bins for all of them 57).
// Many rows are bound by the exponential's instructions (512 rows of 131072 in bf16: 56 us, 48 of them the parts' sums, 2.8 TB/s), few by the launches, each
// a chain of some 2 us accesses to memory with a workgroup's work between them (one row of 131072 in float32 with top_p: 32 us; without filters, two
// launches, 13).
// A row whose list would be too long (thousands of like logits at the cut, a top_k of thousands) is cut by its last workgroup alone, in passes over the row: 131072
// equal logits in float32 with top_p 620 us, with top_k 370, a top_k of 4000 138 (48 such rows: 666, 381, 157).
#include "sample_tokens.h"

#include <type_traits>

#include "token_ops.h"

namespace rlkv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 4096;
constexpr float kBinsPerUnit = 128.f;     // bins: the way from the largest logit over the temperature, 32 of it
constexpr int kList = 2048;               // tokens of a row's list
constexpr int kCompared = 256;            // tokens of a list that are compared with each other; more are sorted (27 rows, 1000 of 38416: 46 us, compared 228)
constexpr int kPart = 8192;               // tokens of a part
constexpr int kChunks = 64;               // of a part, of 128 tokens, eight in each of 16 lanes: their largest logits are kept
constexpr int kSums = kWaves;             // of a part, of 512 tokens: the weights above the list's
constexpr int kMostGroups = 256;          // groups of chunks whose largest logits are ranked
constexpr int kFewThreads = 256;          // of the launches that many rows have many workgroups of
constexpr int kRowsAtOnce = 512;          // rows that have a workspace

// Ascending with x; zeros of either sign are the same.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
template <int CTRL, typename T>
__device__ __forceinline__ T turned(T x) {
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
  const uint32_t low = __builtin_amdgcn_update_dpp(0, (uint32_t)b, CTRL, 0xf, 0xf, false), high = __builtin_amdgcn_update_dpp(0, (uint32_t)(b >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(T, (unsigned long long)high << 32 | low);
}
// Largest of each 16 lanes.
__device__ __forceinline__ float max_of_16(float x) {
  auto step = [&](auto ctrl) {
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  step(std::integral_constant<int, 0xb1>{});
  step(std::integral_constant<int, 0x4e>{});
  step(std::integral_constant<int, 0x141>{});
  step(std::integral_constant<int, 0x140>{});
  return x;
}
template <typename T>
__device__ __forceinline__ T lane_of(T x, int lane) {
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
  const uint32_t low = __builtin_amdgcn_readlane((uint32_t)b, lane), high = __builtin_amdgcn_readlane((uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(T, (unsigned long long)high << 32 | low);
}
// In the registers (neighbours, pairs, the halves and the whole of 16 lanes mirrored, the four rows of 16), the same in all lanes; all have to be there.
template <typename T>
__device__ __forceinline__ T sum_over_wave(T x) {
  x += turned<0xb1>(x);
  x += turned<0x4e>(x);
  x += turned<0x141>(x);
  x += turned<0x140>(x);
  return (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
}

// 2^(j / 128)
constexpr int kRootCount = 128;
__constant__ double kRoots[kRootCount] = {
    0x1.0000000000000p+0, 0x1.0163da9fb3335p+0, 0x1.02c9a3e778061p+0, 0x1.04315e86e7f85p+0,
    0x1.059b0d3158574p+0, 0x1.0706b29ddf6dep+0, 0x1.0874518759bc8p+0, 0x1.09e3ecac6f383p+0,
    0x1.0b5586cf9890fp+0, 0x1.0cc922b7247f7p+0, 0x1.0e3ec32d3d1a2p+0, 0x1.0fb66affed31bp+0,
    0x1.11301d0125b51p+0, 0x1.12abdc06c31ccp+0, 0x1.1429aaea92de0p+0, 0x1.15a98c8a58e51p+0,
    0x1.172b83c7d517bp+0, 0x1.18af9388c8deap+0, 0x1.1a35beb6fcb75p+0, 0x1.1bbe084045cd4p+0,
    0x1.1d4873168b9aap+0, 0x1.1ed5022fcd91dp+0, 0x1.2063b88628cd6p+0, 0x1.21f49917ddc96p+0,
    0x1.2387a6e756238p+0, 0x1.251ce4fb2a63fp+0, 0x1.26b4565e27cddp+0, 0x1.284dfe1f56381p+0,
    0x1.29e9df51fdee1p+0, 0x1.2b87fd0dad990p+0, 0x1.2d285a6e4030bp+0, 0x1.2ecafa93e2f56p+0,
    0x1.306fe0a31b715p+0, 0x1.32170fc4cd831p+0, 0x1.33c08b26416ffp+0, 0x1.356c55f929ff1p+0,
    0x1.371a7373aa9cbp+0, 0x1.38cae6d05d866p+0, 0x1.3a7db34e59ff7p+0, 0x1.3c32dc313a8e5p+0,
    0x1.3dea64c123422p+0, 0x1.3fa4504ac801cp+0, 0x1.4160a21f72e2ap+0, 0x1.431f5d950a897p+0,
    0x1.44e086061892dp+0, 0x1.46a41ed1d0057p+0, 0x1.486a2b5c13cd0p+0, 0x1.4a32af0d7d3dep+0,
    0x1.4bfdad5362a27p+0, 0x1.4dcb299fddd0dp+0, 0x1.4f9b2769d2ca7p+0, 0x1.516daa2cf6642p+0,
    0x1.5342b569d4f82p+0, 0x1.551a4ca5d920fp+0, 0x1.56f4736b527dap+0, 0x1.58d12d497c7fdp+0,
    0x1.5ab07dd485429p+0, 0x1.5c9268a5946b7p+0, 0x1.5e76f15ad2148p+0, 0x1.605e1b976dc09p+0,
    0x1.6247eb03a5585p+0, 0x1.6434634ccc320p+0, 0x1.6623882552225p+0, 0x1.68155d44ca973p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6c012750bdabfp+0, 0x1.6dfb23c651a2fp+0, 0x1.6ff7df9519484p+0,
    0x1.71f75e8ec5f74p+0, 0x1.73f9a48a58174p+0, 0x1.75feb564267c9p+0, 0x1.780694fde5d3fp+0,
    0x1.7a11473eb0187p+0, 0x1.7c1ed0130c132p+0, 0x1.7e2f336cf4e62p+0, 0x1.80427543e1a12p+0,
    0x1.82589994cce13p+0, 0x1.8471a4623c7adp+0, 0x1.868d99b4492edp+0, 0x1.88ac7d98a6699p+0,
    0x1.8ace5422aa0dbp+0, 0x1.8cf3216b5448cp+0, 0x1.8f1ae99157736p+0, 0x1.9145b0b91ffc6p+0,
    0x1.93737b0cdc5e5p+0, 0x1.95a44cbc8520fp+0, 0x1.97d829fde4e50p+0, 0x1.9a0f170ca07bap+0,
    0x1.9c49182a3f090p+0, 0x1.9e86319e32323p+0, 0x1.a0c667b5de565p+0, 0x1.a309bec4a2d33p+0,
    0x1.a5503b23e255dp+0, 0x1.a799e1330b358p+0, 0x1.a9e6b5579fdbfp+0, 0x1.ac36bbfd3f37ap+0,
    0x1.ae89f995ad3adp+0, 0x1.b0e07298db666p+0, 0x1.b33a2b84f15fbp+0, 0x1.b59728de5593ap+0,
    0x1.b7f76f2fb5e47p+0, 0x1.ba5b030a1064ap+0, 0x1.bcc1e904bc1d2p+0, 0x1.bf2c25bd71e09p+0,
    0x1.c199bdd85529cp+0, 0x1.c40ab5fffd07ap+0, 0x1.c67f12e57d14bp+0, 0x1.c8f6d9406e7b5p+0,
    0x1.cb720dcef9069p+0, 0x1.cdf0b555dc3fap+0, 0x1.d072d4a07897cp+0, 0x1.d2f87080d89f2p+0,
    0x1.d5818dcfba487p+0, 0x1.d80e316c98398p+0, 0x1.da9e603db3285p+0, 0x1.dd321f301b460p+0,
    0x1.dfc97337b9b5fp+0, 0x1.e264614f5a129p+0, 0x1.e502ee78b3ff6p+0, 0x1.e7a51fbc74c83p+0,
    0x1.ea4afa2a490dap+0, 0x1.ecf482d8e67f1p+0, 0x1.efa1bee615a27p+0, 0x1.f252b376bba97p+0,
    0x1.f50765b6e4540p+0, 0x1.f7bfdad9cbe14p+0, 0x1.fa7c1819e90d8p+0, 0x1.fd3c22b8f71f1p+0};

// The weight of a logit: 2^bits exp((x - ref) / t), rounded to a whole number.
// With z = 128 log2(e) (x - ref) / t = 128 n + j + r, |r| <= 1/2:  2^n 2^(j / 128) (1 + a r + .. + (a r)^3 / 6), a = ln(2) / 128: the series ends 2.3e-12 of
// it.  Fourteen instructions, which is what the launch over many rows is bound by.
struct Weight {
  const uint64_t* roots;     // in LDS, times 2^bits; j / 128 less in the exponent, to which k / 128 is added with its fraction
  double ref, c;             // 128 log2(e) / t, not 0: at an infinite temperature what is masked keeps its distance
  double lowest;             // of x - ref, where z is -128 (bits + 600): what is below it, or masked (a place of -infinity), has 2^-600
  double least;              // least weight that counts, of 2^bits (min_p)
  __device__ __forceinline__ double real(float x) const {
    const double way = fmax((double)x - ref, lowest);
    const double shifted = __builtin_fma(way, c, 6755399441055744.);        // 1.5 * 2^52: the nearest whole number in the low bits
    const uint32_t k = (uint32_t)__double_as_longlong(shifted);
    const double r = __builtin_fma(way, c, -(shifted - 6755399441055744.));
    constexpr double a = 0.69314718055994530942 / kRootCount;
    double p = __builtin_fma(r, a * a * a / 6, a * a / 2);
    p = __builtin_fma(r, p, a);
    p = __builtin_fma(r, p, 1.);
    typedef uint32_t words __attribute__((ext_vector_type(2)));
    words root = __builtin_bit_cast(words, roots[k & (kRootCount - 1)]);
    root.y += k << 13;
    return __builtin_bit_cast(double, root) * p;
  }
  __device__ __forceinline__ unsigned long long rounded(double w) const {       // (by adding 2^52)
    return (unsigned long long)__double_as_longlong(w + 4503599627370496.) - 0x4330000000000000ull;
  }
  __device__ __forceinline__ unsigned long long operator()(float x) const {
    const double w = real(x);
    return w >= least ? rounded(w) : 0;
  }
  __device__ __forceinline__ unsigned long long whole(float x) const { return rounded(real(x)); }      // without min_p
};
// (w below 2^51: bits is at most 50 then)
__host__ __device__ inline int bits_of(int vocab) {
  int bits = 62;
  for (int64_t n = 1; n < vocab; n *= 2) --bits;
  return bits < 50 ? bits : 50;
}

// The share of a sum of weights that is to be reached: whole weights reach it where they reach the next whole number.
__device__ __forceinline__ unsigned long long whole_share(double p, double total) { return (unsigned long long)ceil(p * total); }

struct Settings {
  double t, top_p, min_p;
  int top_k;                 // 0: off, and so where it is no less than vocab
  __device__ bool greedy() const { return !(t > 0.); }
  __device__ bool cut() const { return !greedy() && (top_k > 0 || top_p < 1.); }
  __device__ bool filter() const { return cut() || (!greedy() && min_p > 0.); }
};
__device__ __forceinline__ Settings settings_of(const SampleCall& c, int64_t n) {
  Settings s;
  s.t = c.temperatures ? c.temperatures[n] : c.temperature;
  s.top_p = c.top_ps ? c.top_ps[n] : c.top_p;
  s.min_p = c.min_ps ? c.min_ps[n] : c.min_p;
  s.top_k = c.top_ks ? c.top_ks[n] : c.top_k;
  if (s.top_k >= c.vocab || s.top_k < 0) s.top_k = 0;
  if (!(s.top_p < 1.)) s.top_p = 1.;
  if (s.top_p < 0.) s.top_p = 0.;
  s.min_p = s.min_p > 0. ? (s.min_p < 1. ? s.min_p : 1.) : 0.;
  return s;
}
// (1 / t is at most 1e300: a way of 0 stays 0)
__device__ __forceinline__ double inverse(double t) { return t > 1e-300 ? 1. / t : 1e300; }
__device__ __forceinline__ Weight weight_of(const Settings& s, const uint64_t* roots, double ref, int bits, double least) {
  const double c = fmax(inverse(s.t), 1e-250) * (kRootCount * 1.4426950408889634074);
  return {roots, ref, c, -1. * kRootCount * (bits + 600) / c, least};
}

// Steps down from the largest logit; not decreasing as x falls.
struct FirstBin {
  float top, per;
  __device__ __forceinline__ int operator()(float x) const {
    const float z = (top - x) * per;
    return z < (float)(kBins - 1) ? (int)z : kBins - 1;       // (NaN, of a masked logit at an infinite temperature: the last)
  }
};
__device__ __forceinline__ FirstBin first_bin(float top, const Settings& s) { return {top, fminf((float)inverse(s.t) * kBinsPerUnit, 3e38f)}; }      // (no infinity: 0 times it)

// ---- the workspace ----
struct Part {
  float top;
  int32_t bad;                     // a NaN or +inf is there
  double sum;                      // of weights with the part's largest logit for reference, of 2^bits
  unsigned long long above;        // of weights above the list's that min_p keeps, with the row's largest for reference
};
struct RowCut {
  int32_t listed;                  // tokens of the list; more than kList: there is no list
  uint32_t by_tops;                // the list is made by the last launch
  unsigned long long before;       // weight of the tokens above the list's
};
struct RowSpace {
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  unsigned long long list[kList];  // ~key, token: ascending is the order of the cut
  RowCut cut;
};
struct Space {
  RowSpace* rows;
  Part* parts;                     // [rows][n_parts]
  unsigned long long* sums;        // [rows][n_parts][kSums]
  float* tops;                     // [rows][n_parts][kChunks]
  int32_t n_parts;
  int64_t first_row;               // of the launch
};

struct PlaceSmem {
  unsigned long long sums[kWaves];
  int32_t index;
};
struct Smem {
  PlaceSmem place;
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  unsigned long long sums[kWaves];
  uint32_t low[kWaves], high[kWaves];
  unsigned long long found_before, found_mass;
  uint32_t found, found_count;
  int32_t index;
  uint64_t roots[kRootCount];
};

// What is kept: keys above `key`, and `key` itself up to the place `last`.
struct Row {
  float top;
  Settings how;
  uint32_t key;
  int32_t last;
};
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

// First place in [lo, hi) where the running sum of f is above `target`, in all threads; where there is none, the last one where f is above 0 (one
// there has to be).
template <int THREADS, typename T, typename F>
__device__ __forceinline__ int place_of(PlaceSmem& sm, const T* row, int lo, int hi, unsigned long long target, F f) {
  constexpr int kWaves = THREADS / 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  while (hi - lo > THREADS * 8) {            // a part for each wavefront
    const int part = ((hi - lo + kWaves - 1) / kWaves + 7) / 8 * 8;
    const int64_t a = lo + (int64_t)wave * part, b = a + part;
    unsigned long long sum = 0;
    if (a < hi) each_token(row, (int)a, (int)(b < hi ? b : hi), lane, 64, [&](float x, int i) { sum += f(x, i); });
    sum = sum_over_wave(sum);
    __syncthreads();
    if (lane == 0) sm.sums[wave] = sum;
    __syncthreads();
    int found = 0;
    bool inside = false;
    for (int w = 0; w < kWaves && !inside; ++w) {
      const unsigned long long s = sm.sums[w];
      if (s == 0) continue;
      found = w;
      inside = target < s;
      if (!inside) target -= s;
    }
    if (!inside) target = ~0ull >> 1;        // (behind all sums that follow, too)
    lo += found * part;
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
  if (threadIdx.x == 0) sm.index = -1;
  __syncthreads();
  before -= sum;
  unsigned long long total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sm.sums[w];
    total += sm.sums[w];
  }
  if (target >= total) target = total - 1;   // (the last token's share)
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
__device__ __forceinline__ void bin_of(Smem& sm, bool by_mass, unsigned long long target) {
  constexpr int kEach = kBins / kThreads;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = threadIdx.x * kEach;
  unsigned long long v[kEach], own = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = by_mass ? sm.mass[first + i] : sm.count[first + i];
    own += v[i];
  }
  unsigned long long run = own;
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long other = __shfl_up(run, d);
    if (lane >= d) run += other;
  }
  if (lane == 63) sm.sums[wave] = run;
  __syncthreads();
  run -= own;
  for (int w = 0; w < wave; ++w) run += sm.sums[w];
  if (run <= target && target < run + own) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (run <= target && target < run + v[i]) {
        sm.found = first + i;
        sm.found_before = run;
        sm.found_mass = sm.mass[first + i];
        sm.found_count = sm.count[first + i];
      }
      run += v[i];
    }
  }
  __syncthreads();
}

// Cuts the kept tokens of `r` to the first ones in order of their logits: to `target` of them, or (by_mass) to those in front of which the weights
// sum to less than `target`.  There are more of them.
template <typename T>
__device__ __forceinline__ void cut(Smem& sm, const T* row, int vocab, Row& r, const Weight& weight, bool by_mass, unsigned long long target) {
  const FirstBin bin_at = first_bin(r.top, r.how);
  auto add = [&](int bin, float x) {
    atomicAdd(&sm.count[bin], 1u);
    if (by_mass) {
      const unsigned long long w = weight(x);
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
    if (keeps(r, x, i)) add(bin_at(x), x);
  });
  __syncthreads();
  bin_of(sm, by_mass, last);
  const int bin = sm.found;
  unsigned long long before = sm.found_before;
  // the keys of that bin, and by them bins of fewer and fewer keys
  uint32_t low = 0xffffffffu, high = 0;
  each_token(row, 0, vocab, threadIdx.x, kThreads, [&](float x, int i) {
    if (bin_at(x) != bin || !keeps(r, x, i)) return;
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
  if (need < count) place = place_of<kThreads>(sm.place, row, 0, vocab, need - 1, [&](float x, int i) { return (unsigned long long)(key_of(x) == high && i <= old_last); });
  r.key = high;
  r.last = place;
}

// ---- the launches ------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void load_roots(uint64_t* roots, int bits) {
  if (threadIdx.x < kRootCount) roots[threadIdx.x] = (uint64_t)__double_as_longlong(kRoots[threadIdx.x]) + ((uint64_t)bits << 52) - ((uint64_t)threadIdx.x << 45);
}
// What a row's parts (a few dozen) come to, in every wavefront that asks: lane l reads the parts l, l + 64, ..
struct RowParts {
  const Part* parts;
  int n;
  struct { float top; double sum; } first;      // of this lane
  float top;                       // the row's largest logit
  bool drawn;                      // there is something to draw from
  __device__ __forceinline__ RowParts(const Part* parts, int n) : parts(parts), n(n) {
    const int lane = threadIdx.x & 63;
    const Part& part = parts[lane < n ? lane : 0];
    first = {part.top, part.sum};
    top = first.top;
    bool bad = part.bad != 0;
    for (int p = lane + 64; p < n; p += 64) {
      top = fmaxf(top, parts[p].top);
      bad |= parts[p].bad != 0;
    }
    top = max_of_wave(top);
    drawn = !__any(bad) && top != -INFINITY;
  }
  // Sum of the row's weights with `top` for reference, of 2^bits: parts in a fixed order.
  __device__ __forceinline__ double total(double inv) const {
    const int lane = threadIdx.x & 63;
    double sum = lane < n && first.top != -INFINITY ? first.sum * exp(((double)first.top - (double)top) * inv) : 0.;
    for (int p = lane + 64; p < n; p += 64)
      if (parts[p].top != -INFINITY) sum += parts[p].sum * exp(((double)parts[p].top - (double)top) * inv);
    return sum_over_wave(sum);
  }
};

// The tokens of a part, all asked for at once; -infinity behind the row's end.
template <typename T, int THREADS>
struct PartTokens {
  static constexpr int PIECES = kPart / 8 / THREADS;
  float x[PIECES][8];
  int lo;
  __device__ __forceinline__ PartTokens(const T* row, int part, int vocab) : lo(part * kPart) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const int at = place(k);
      if (at + 8 <= vocab) {
        widen(piece_at<false>(row + at), x[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[k][i] = at + i < vocab ? one_value(row[at + i]) : -INFINITY;
      }
    }
  }
  __device__ __forceinline__ int place(int k) const { return lo + (k * THREADS + (int)threadIdx.x) * 8; }
  template <typename F>
  __device__ __forceinline__ void each(int vocab, F f) const {
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (place(k) + i < vocab) f(x[k][i], place(k) + i);
  }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void parts_kernel(SampleCall c, Space space, int bits, int cuts) {
  constexpr int kWaves = THREADS / 64, PIECES = kPart / 8 / THREADS;
  __shared__ uint64_t roots[kRootCount];
  __shared__ float tops[kWaves];
  __shared__ double sums[kWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, p = blockIdx.x;
  const int64_t n = space.first_row + blockIdx.y;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  const PartTokens<T, THREADS> part(row, p, c.vocab);
  const auto& x = part.x;
  const Settings s = settings_of(c, n);
  load_roots(roots, bits);
  // (what the next launches add up starts at 0)
  if (cuts && s.cut()) {
    RowSpace& r = space.rows[blockIdx.y];
    for (int b = p * THREADS + threadIdx.x; b < kBins; b += space.n_parts * THREADS) {
      r.mass[b] = 0;
      r.count[b] = 0;
    }
    if (p == 0 && threadIdx.x == 0) {
      r.cut.listed = 0;
      r.cut.by_tops = 0;
    }
  }
  Part& result = space.parts[(int64_t)blockIdx.y * space.n_parts + p];
  float top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    float here = x[k][0];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      here = fmaxf(here, x[k][i]);
      bad |= !(x[k][i] < INFINITY);
    }
    if (cuts) {
      here = max_of_16(here);
      if (lane % 16 == 0) space.tops[((int64_t)blockIdx.y * space.n_parts + p) * kChunks + (k * THREADS + threadIdx.x) / 16] = here;
    }
    top = fmaxf(top, here);
  }
  top = max_of_wave(top);
  if (lane == 0) tops[wave] = top;
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
  double sum = 0.;
  // (a top_k's weights are those of its list, and what min_p alone keeps is summed later)
  if (!bad && top != -INFINITY && !s.greedy() && s.top_k == 0 && (s.top_p < 1. || !s.filter())) {
    const Weight weight = weight_of(s, roots, top, bits, 0.);
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += weight.real(x[k][i]);
    sum = sum_over_wave(sum);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sums[w];
  }
  if (threadIdx.x == 0) {
    result.top = top;
    result.bad = bad;
    result.sum = sum;
    result.above = 0;
  }
}

// The rule by which a row's top_k is found among the largest logits of groups of chunks: the k-th largest of n of them is reached by k tokens at
// least and by some n ln(n / (n - k)) where tokens lie in no order, 1.4 n for the largest k, three quarters of n: the list has room.  A row of 128k tokens
// that wants 50 lists 53.
struct Groups {
  int each, n;                     // chunks of a group, groups
  __device__ __forceinline__ Groups(int n_parts, int vocab) {
    each = (n_parts * kChunks + kMostGroups - 1) / kMostGroups;
    n = vocab < 8 ? 0 : (n_parts * kChunks + each - 1) / each;      // (the list is made from eight tokens at a time)
  }
  __device__ __forceinline__ bool serve(int top_k) const { return top_k > 0 && 4 * (int64_t)top_k <= 3 * (int64_t)n; }
  // of this thread's group, -infinity for what is none
  __device__ __forceinline__ float top(const float* tops, int n_parts) const {
    float most = -INFINITY;
    if ((int)threadIdx.x < n)
      for (int i = threadIdx.x * each; i < min(((int)threadIdx.x + 1) * each, n_parts * kChunks); ++i) most = fmaxf(most, tops[i]);
    return most;
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads, 8) void bins_kernel(SampleCall c, Space space, int bits) {
  __shared__ uint64_t roots[kRootCount];
  __shared__ unsigned long long mass[kBins];
  __shared__ uint32_t count[kBins];
  const int64_t n = space.first_row + blockIdx.y;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  const Settings s = settings_of(c, n);
  if (!s.cut()) return;
  const Part* parts = space.parts + (int64_t)blockIdx.y * space.n_parts;
  const Groups groups(space.n_parts, c.vocab);
  if (groups.serve(s.top_k)) {
    const float most = groups.top(space.tops + (int64_t)blockIdx.y * space.n_parts * kChunks, space.n_parts);
    // (of tokens masked nearly everywhere there are too few groups to rank)
    if (__syncthreads_count(most != -INFINITY) >= s.top_k) {
      if (blockIdx.x == 0 && threadIdx.x == 0) space.rows[blockIdx.y].cut.by_tops = 1;
      return;
    }
  }
  const PartTokens<T, kThreads> part(row, blockIdx.x, c.vocab);      // (asked for before anything is waited for)
  load_roots(roots, bits);
  const RowParts all(parts, space.n_parts);
  if (!all.drawn) return;
  const float top = all.top;
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    mass[b] = 0;
    count[b] = 0;
  }
  __syncthreads();
  const FirstBin bin_at = first_bin(top, s);
  const Weight weight = weight_of(s, roots, top, bits, 0.);
  const bool by_mass = s.top_k == 0;
  // Tokens that top_p keeps for sure not: those of a weight below (1 - p) sum / vocab have less than 1 - p of the sum together.
  unsigned long long least = 0;
  if (by_mass) {
    least = (unsigned long long)((1. - s.top_p) * all.total(inverse(s.t)) * 0.99 / c.vocab);
  }
  part.each(c.vocab, [&](float x, int) {
    const int b = bin_at(x);
    if (by_mass) {
      const unsigned long long w = weight.whole(x);
      if (w < least || w == 0) return;
      atomicAdd(&mass[b], w);
    }
    atomicAdd(&count[b], 1u);
  });
  __syncthreads();
  RowSpace& r = space.rows[blockIdx.y];
  for (int b = threadIdx.x; b < kBins; b += kThreads) {
    if (count[b]) atomicAdd(&r.count[b], count[b]);
    if (mass[b]) atomicAdd(&r.mass[b], mass[b]);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads, 8) void collect_kernel(SampleCall c, Space space, int bits) {
  __shared__ uint64_t roots[kRootCount];
  __shared__ unsigned long long sums[kWaves];
  __shared__ int32_t found, found_count, here, at_list;
  __shared__ unsigned long long found_before, list[kList];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t n = space.first_row + blockIdx.y;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  Part* parts = space.parts + (int64_t)blockIdx.y * space.n_parts;
  const Settings s = settings_of(c, n);
  RowSpace& r = space.rows[blockIdx.y];
  if (!s.filter() || (s.cut() && s.top_k > 0 && r.cut.by_tops)) return;
  // (all of it asked for before anything is waited for)
  const PartTokens<T, kThreads> part(row, blockIdx.x, c.vocab);
  constexpr int kEach = kBins / kThreads;
  const bool by_mass = s.top_k == 0;
  unsigned long long v[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) v[i] = !s.cut() ? 0 : by_mass ? r.mass[threadIdx.x * kEach + i] : r.count[threadIdx.x * kEach + i];
  load_roots(roots, bits);
  const RowParts all(parts, space.n_parts);
  if (!all.drawn) return;
  const float top = all.top;
  int first = kBins, last = kBins;                  // bins [first, last] are listed
  if (s.cut()) {
    const unsigned long long target = by_mass ? whole_share(s.top_p, all.total(inverse(s.t))) : 0;
    unsigned long long run = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) run += v[i];
    const unsigned long long own = run;
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned long long other = __shfl_up(run, d);
      if (lane >= d) run += other;
    }
    if (lane == 63) sums[wave] = run;
    if (threadIdx.x == 0) found = kBins;
    __syncthreads();
    run -= own;
    for (int w = 0; w < wave; ++w) run += sums[w];
    // the bin that reaches the target (the first with any weight, where the target is 0)
    auto reached = [&](unsigned long long x) { return by_mass ? x > 0 && x >= target : x >= (unsigned long long)s.top_k; };
    if (!reached(run)) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (reached(run + v[i]) && !reached(run)) {
          found = threadIdx.x * kEach + i;
          found_count = (int)(by_mass ? r.count[threadIdx.x * kEach + i] : run + v[i]);
          found_before = run;
        }
        run += v[i];
      }
    }
    __syncthreads();
    last = found;
    first = by_mass ? last : 0;
    if (last < kBins && blockIdx.x == 0 && threadIdx.x == 0) {
      r.cut.before = by_mass ? found_before : 0;
      if (found_count > kList) atomicAdd(&r.cut.listed, kList + 1);
    }
    // (none reaches it, by the roundings of the target: nothing is cut)
    if (last < kBins && found_count > kList) return;
  }
  if (threadIdx.x == 0) here = 0;
  __syncthreads();
  const FirstBin bin_at = first_bin(top, s);
  const Weight weight = weight_of(s, roots, top, bits, s.min_p * (double)(1ull << bits));
  unsigned long long sum = 0;
  part.each(c.vocab, [&](float x, int i) {
    const int b = first == kBins ? 0 : bin_at(x);
    if (b < first) {
      sum += weight(x);
    } else if (b <= last) {
      const int at = atomicAdd(&here, 1);
      if (at < kList) list[at] = (unsigned long long)~key_of(x) << 32 | (uint32_t)i;
    }
  });
  sum = sum_over_wave(sum);
  __syncthreads();
  if (lane == 0) {
    sums[wave] = sum;
    space.sums[((int64_t)blockIdx.y * space.n_parts + blockIdx.x) * kSums + wave] = sum;
  }
  if (threadIdx.x == 0 && here > 0) at_list = atomicAdd(&r.cut.listed, here);
  __syncthreads();
  for (int j = threadIdx.x; j < here && at_list + j < kList; j += kThreads) r.list[at_list + j] = list[j];
  if (threadIdx.x == 0) {
    sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sums[w];
    parts[blockIdx.x].above = sum;
  }
}

// The part that a row's number falls into where there are no filters: parts have references of their own, so their sums are added in 64-bit floating
// point, in a fixed order.  One wavefront; part, way into it, sum of the row.
struct PlainDraw {
  double total;
  unsigned long long way;
  int32_t part;
};
__device__ __forceinline__ PlainDraw plain_part(const RowParts& all, double inv, float u) {
  const Part* parts = all.parts;
  const int n = all.n;
  const float top = all.top;
  const int lane = threadIdx.x & 63;
  double run = 0., before = 0.;
  int found = -1;
  auto weight_at = [&](int p) { return p < n && parts[p].top != -INFINITY ? parts[p].sum * exp(((double)parts[p].top - (double)top) * inv) : 0.; };
  const double total = all.total(inv);
  const double target = (u > 0.f ? u < 1.f ? (double)u : 1. - 1e-16 : 0.) * total;
  for (int p0 = 0; p0 < n; p0 += 64) {
    const double w = weight_at(p0 + lane);
    double upto = w;
    for (int d = 1; d < 64; d <<= 1) {
      const double other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    upto += run;
    run = __shfl(upto, 63);
    // the first one past the target; by the roundings of the sums there may be none: the last with any weight
    const unsigned long long past = __ballot(w > 0. && target < upto), any = __ballot(w > 0.);
    if (!any) continue;
    const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
    found = p0 + at;
    before = __shfl(upto - w, at);
    if (past) break;
  }
  // (the way into the part, in its own unit; where the roundings of the sums lead behind the part's last token, that one is drawn)
  const double way = (target - before) / exp(((double)parts[found].top - (double)top) * inv);
  return {total, way > 0. ? (unsigned long long)way : 0, found};
}

// Rows without filters, the temperature the same for all and above 0.
template <typename T>
__global__ __launch_bounds__(kFewThreads) void draw_plain_kernel(SampleCall c, Space space, int bits) {
  __shared__ PlaceSmem place;
  __shared__ uint64_t roots[kRootCount];
  const int64_t n = space.first_row + blockIdx.x;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  const Part* parts = space.parts + (int64_t)blockIdx.x * space.n_parts;
  Settings s = {c.temperature, 1., 0., 0};
  const float u = c.uniforms[n];
  const RowParts all(parts, space.n_parts);
  const float top = all.top;
  if (!all.drawn) {                                     // nothing to draw from
    if (threadIdx.x == 0) {
      c.tokens[n] = -1;
      if (c.logprobs) c.logprobs[n] = NAN;
    }
    return;
  }
  load_roots(roots, bits);
  const double inv = inverse(s.t);
  const PlainDraw d = plain_part(all, inv, u);      // (every wavefront for itself)
  const Weight weight = weight_of(s, roots, parts[d.part].top, bits, 0.);
  const int lo = d.part * kPart;
  __syncthreads();
  const int i = place_of<kFewThreads>(place, row, lo, min(lo + kPart, c.vocab), d.way, [&](float x, int) { return weight.whole(x); });
  if (threadIdx.x == 0) {
    c.tokens[n] = i;
    if (c.logprobs) c.logprobs[n] = (float)(((double)one_value(row[i]) - (double)top) * inv - log(d.total / (double)(1ull << bits)));
  }
}

// Of up to kCompared tokens this thread's: the one that it compares and those that it is compared with.
struct Share {
  int j, from, to;
  __device__ __forceinline__ explicit Share(int count) {
    int each = 64;
    while (each < count) each *= 2;
    const int len = (count + kThreads / each - 1) / (kThreads / each);
    j = threadIdx.x % each;
    from = threadIdx.x / each * len;
    to = min(from + len, count);
  }
};
// Ascending; size, a power of two, twice the workgroup's threads at most.  Bitonic: steps over less than 128 places are a wavefront's own.
__device__ __forceinline__ void sort(unsigned long long* x, int size) {
  const int t = threadIdx.x;
#pragma unroll 1
  for (int run = 2; run <= size; run *= 2)
#pragma unroll 1
    for (int step = run / 2; step; step /= 2) {
      if (t < size / 2) {
        const int a = 2 * (t & -step) + (t & (step - 1)), b = a + step;
        const unsigned long long low = x[a], high = x[b];
        if ((low > high) == ((a & run) == 0)) {
          x[a] = high;
          x[b] = low;
        }
      }
      if (step > 64 || (step == 1 && run > 64)) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  __syncthreads();
}
// The list of a row that is cut by top_k, made from the chunks that reach the top_k-th largest of the groups' largest logits; its length, which may be
// more than kList (then there is no list).
template <typename T>
__device__ __forceinline__ int list_by_tops(Smem& sm, unsigned long long* list, const T* row, int vocab, const float* tops, int n_parts, const Groups& groups, float most, int top_k) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = groups.n;
  uint32_t *keys = sm.count, *chunks = keys + kMostGroups;
  if ((int)threadIdx.x < kMostGroups) keys[threadIdx.x] = (int)threadIdx.x < n ? key_of(most) : 0;
  if (threadIdx.x == 0) {
    sm.found_count = 0;
    sm.index = 0;
  }
  __syncthreads();
  // the largest key that top_k of them reach, two bits at a time: one wavefront (comparing all with all took ten times as long)
  if (wave == 0) {
    uint32_t key[kMostGroups / 64], reached = 0;
#pragma unroll
    for (int i = 0; i < kMostGroups / 64; ++i) key[i] = keys[64 * i + lane];
#pragma unroll 1
    for (int shift = 30; shift >= 0; shift -= 2) {
      int count[4] = {};
#pragma unroll
      for (int i = 0; i < kMostGroups / 64; ++i)
#pragma unroll
        for (int d = 1; d < 4; ++d) count[d] += __popcll(__ballot(key[i] >= (reached | (uint32_t)d << shift)));
      reached |= (uint32_t)((count[1] >= top_k) + (count[2] >= top_k) + (count[3] >= top_k)) << shift;
    }
    if (lane == 0) sm.found = reached;
  }
  __syncthreads();
  const uint32_t bound = sm.found;
  for (int i = threadIdx.x; i < n_parts * kChunks; i += kThreads)
    if (key_of(tops[i]) >= bound) {
      const uint32_t at = atomicAdd(&sm.found_count, 1u);
      if (at < kList) chunks[at] = i;
    }
  __syncthreads();
  const int hit = sm.found_count;
  if (hit > kList) return hit;
  constexpr int kAtOnce = 2, kHere = 64 / (kPart / kChunks / 8);      // pieces of a lane asked for together; chunks of a wavefront's piece
  for (int c = wave * kAtOnce * kHere; c < hit; c += kWaves * kAtOnce * kHere) {
    // (the last lanes of a row read its last eight tokens and take their own of them: no branches, the loads go out together)
    float x[kAtOnce][8];
    int at[kAtOnce], first[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int chunk = c + q * kHere + lane / (64 / kHere);
      at[q] = chunk < hit ? (int)chunks[chunk] * (kPart / kChunks) + lane % (64 / kHere) * 8 : vocab;
      first[q] = min(at[q], vocab - 8);
      widen(piece_at<false>(row + first[q]), x[q]);
    }
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      uint32_t reach = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) reach |= (uint32_t)(first[q] + i >= at[q] && key_of(x[q][i]) >= bound) << i;
      if (reach == 0) continue;
      int slot = atomicAdd(&sm.index, __popc(reach));
      for (; reach; reach &= reach - 1, ++slot) {
        const int which = __builtin_ctz(reach);
        float v = x[q][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) v = which == i ? x[q][i] : v;
        if (slot < kList) list[slot] = (unsigned long long)~key_of(v) << 32 | (uint32_t)(first[q] + which);
      }
    }
  }
  __syncthreads();
  const int listed = sm.index;
  __syncthreads();
  return listed;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void draw_kernel(SampleCall c, Space space, int bits) {
  __shared__ Smem sm;
  const int64_t n = space.first_row + blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T* row = static_cast<const T*>(c.logits) + n * c.stride;
  const Part* parts = space.parts + (int64_t)blockIdx.x * space.n_parts;
  RowSpace& space_of_row = space.rows[blockIdx.x];
  const float* tops = space.tops + (int64_t)blockIdx.x * space.n_parts * kChunks;
  Row r;
  r.how = settings_of(c, n);
  r.key = 0;
  r.last = 0x7fffffff;
  const Settings& s = r.how;
  // (what the last launch left, asked for before anything is waited for; behind the list's end it is not used)
  const float u = c.uniforms[n];
  RowCut cut_of_row = {};
  unsigned long long listed_here[kList / kThreads] = {};
  if (s.cut()) {
    cut_of_row = space_of_row.cut;
#pragma unroll
    for (int q = 0; q < kList / kThreads; ++q) listed_here[q] = space_of_row.list[q * kThreads + threadIdx.x];
  }
  const Groups groups(space.n_parts, c.vocab);
  const float most = s.cut() && groups.serve(s.top_k) ? groups.top(tops, space.n_parts) : -INFINITY;
  const RowParts row_parts(parts, space.n_parts);
  r.top = row_parts.top;
  if (!row_parts.drawn) {                               // nothing to draw from
    if (threadIdx.x == 0) {
      c.tokens[n] = -1;
      if (c.logprobs) c.logprobs[n] = NAN;
    }
    return;
  }
  load_roots(sm.roots, bits);
  const double unit = (double)(1ull << bits), inv = inverse(s.t);
  auto write = [&](int i, double total) {
    if (threadIdx.x != 0) return;
    c.tokens[n] = i;
    if (c.logprobs) c.logprobs[n] = (float)(((double)one_value(row[i]) - (double)r.top) * inv - log(total / unit));
  };
  if (s.greedy()) {
    if (threadIdx.x == 0) sm.index = space.n_parts;
    __syncthreads();
    for (int p = threadIdx.x; p < space.n_parts; p += kThreads)
      if (parts[p].top == r.top) atomicMin(&sm.index, p);
    __syncthreads();
    const int lo = sm.index * kPart;
    __syncthreads();
    const int i = place_of<kThreads>(sm.place, row, lo, min(lo + kPart, c.vocab), 0, [&](float x, int) { return (unsigned long long)(x == r.top); });
    if (threadIdx.x == 0) {
      c.tokens[n] = i;
      if (c.logprobs) c.logprobs[n] = 0.f;
    }
    return;
  }
  const unsigned long long u64 = !(u > 0.f) ? 0 : u < 1.f ? (unsigned long long)((double)u * 18446744073709551616.) : ~0ull;
  if (!s.filter()) {
    const PlainDraw d = plain_part(row_parts, inv, u);      // (every wavefront for itself)
    const int p = d.part, lo = p * kPart;
    const Weight weight = weight_of(s, sm.roots, parts[p].top, bits, 0.);
    write(place_of<kThreads>(sm.place, row, lo, min(lo + kPart, c.vocab), d.way, [&](float x, int) { return weight.whole(x); }), d.total);
    return;
  }

  const Weight all = weight_of(s, sm.roots, r.top, bits, 0.), weight = weight_of(s, sm.roots, r.top, bits, s.min_p * unit);
  auto kept_weight = [&](float x, int i) { return keeps(r, x, i) ? weight(x) : 0ull; };
  bool listed = true, list_is_all = false;
  __syncthreads();
  if (s.cut()) {
    unsigned long long* order = sm.mass;                   // (2048 of each)
    if (cut_of_row.by_tops && s.top_k > 0) {
      cut_of_row.listed = list_by_tops(sm, order, row, c.vocab, tops, space.n_parts, groups, most, s.top_k);
      cut_of_row.before = 0;
      list_is_all = true;
#pragma unroll
      for (int q = 0; q < kList / kThreads; ++q) listed_here[q] = order[q * kThreads + threadIdx.x];
    }
    listed = cut_of_row.listed <= kList;
    if (listed && cut_of_row.listed > 0) {
      // every token of the list by how many, and what weight, stand in front of it
      const int count = cut_of_row.listed;
      __shared__ unsigned long long weights[kList];
      __shared__ unsigned long long in_front_of[kList];
      __shared__ uint32_t ahead_of[kList];
      auto weight_of_entry = [&](unsigned long long e) {
        const uint32_t key = ~(uint32_t)(e >> 32);
        return all(__uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key));
      };
      if (count <= kCompared) {
        if ((int)threadIdx.x < count) {
          order[threadIdx.x] = listed_here[0];
          weights[threadIdx.x] = weight_of_entry(listed_here[0]);
          in_front_of[threadIdx.x] = 0;
          ahead_of[threadIdx.x] = 0;
        }
        __syncthreads();
        // (a token's comparisons are shared by as many threads as there are for each)
        const Share mine(count);
        if (mine.j < count) {
          const unsigned long long own = order[mine.j];
          uint32_t ahead = 0;
          unsigned long long sum = 0;
#pragma unroll 8
          for (int i = mine.from; i < mine.to; ++i) {           // (without branches: the reads go out together)
            const bool is = order[i] < own;
            ahead += is;
            sum += is ? weights[i] : 0ull;
          }
          atomicAdd(&ahead_of[mine.j], ahead);
          atomicAdd(&in_front_of[mine.j], sum);
        }
      } else {
        int size = 2 * kCompared;
        while (size < count) size *= 2;
#pragma unroll
        for (int q = 0; q < kList / kThreads; ++q) {
          const int j = q * kThreads + threadIdx.x;
          if (j < size) order[j] = j < count ? listed_here[q] : ~0ull;
        }
        __syncthreads();
        sort(order, size);
        // two neighbours a thread
        unsigned long long own[2], sum = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int j = 2 * threadIdx.x + i;
          own[i] = j < count ? weight_of_entry(order[j]) : 0;
          sum += own[i];
        }
        unsigned long long upto = sum;
        for (int d = 1; d < 64; d <<= 1) {
          const unsigned long long other = __shfl_up(upto, d);
          if (lane >= d) upto += other;
        }
        if (lane == 63) sm.sums[wave] = upto;
        __syncthreads();
        upto -= sum;
        for (int w = 0; w < wave; ++w) upto += sm.sums[w];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int j = 2 * threadIdx.x + i;
          if (j >= count) continue;
          weights[j] = own[i];
          in_front_of[j] = upto;
          ahead_of[j] = j;
          upto += own[i];
        }
#pragma unroll
        for (int q = 0; q < kList / kThreads; ++q) listed_here[q] = q * kThreads + (int)threadIdx.x < count ? order[q * kThreads + threadIdx.x] : 0;
      }
      __syncthreads();
      uint32_t rank[kList / kThreads];
      unsigned long long before[kList / kThreads], mine[kList / kThreads], total = 0;
#pragma unroll
      for (int q = 0; q < kList / kThreads; ++q) {
        const int j = q * kThreads + threadIdx.x;
        rank[q] = 0xffffffffu;
        before[q] = mine[q] = 0;
        if (j >= count) continue;
        mine[q] = order[j];
        rank[q] = ahead_of[j];
        before[q] = in_front_of[j];
        if (s.top_k > 0 && rank[q] < (uint32_t)s.top_k) total += weights[j];
      }
      unsigned long long target = ~0ull;
      if (s.top_p < 1.) {
        if (s.top_k > 0) {
          total = sum_over_wave(total);
          if (lane == 0) sm.sums[wave] = total;
          __syncthreads();
          total = 0;
          for (int w = 0; w < kWaves; ++w) total += sm.sums[w];
          target = whole_share(s.top_p, (double)total);
        } else {
          target = whole_share(s.top_p, row_parts.total(inv));
        }
      }
      if (threadIdx.x == 0) sm.found = 0;
      __syncthreads();
      // the last one that is kept; the most likely one always is
      int keep = -1;
#pragma unroll
      for (int q = 0; q < kList / kThreads; ++q) {
        if (rank[q] == 0xffffffffu || (s.top_k > 0 && rank[q] >= (uint32_t)s.top_k)) continue;
        const unsigned long long in_front = cut_of_row.before + before[q];
        if (in_front == 0 ? rank[q] != 0 : in_front >= target) continue;
        keep = max(keep, (int)rank[q]);
      }
      if (keep >= 0) atomicMax(&sm.found, (uint32_t)keep);
      __syncthreads();
#pragma unroll
      for (int q = 0; q < kList / kThreads; ++q)
        if (rank[q] == sm.found) {
          sm.low[0] = ~(uint32_t)(mine[q] >> 32);
          sm.index = (int32_t)(uint32_t)mine[q];
        }
      __syncthreads();
      r.key = sm.low[0];
      r.last = sm.index;
      __syncthreads();
      if (s.top_k > 0 && count <= kCompared) {
        // all that is kept is in the list: the weight of the kept tokens with lower numbers in front of each
        const int t = threadIdx.x;
        const uint32_t key = ~(uint32_t)(mine[0] >> 32);
        const float x = __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
        const unsigned long long own = t < count ? kept_weight(x, (int)(uint32_t)mine[0]) : 0;
        if (t < count) {
          weights[t] = own;
          in_front_of[t] = 0;
        }
        unsigned long long sum = sum_over_wave(own);
        if (lane == 0) sm.sums[wave] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kWaves; ++w) sum += sm.sums[w];
        const unsigned long long target = __umul64hi(sum, u64);
        const Share part(count);
        if (part.j < count) {
          const uint32_t number = (uint32_t)order[part.j];
          unsigned long long less = 0;
#pragma unroll 8
          for (int i = part.from; i < part.to; ++i) less += (uint32_t)order[i] < number ? weights[i] : 0ull;
          atomicAdd(&in_front_of[part.j], less);
        }
        __syncthreads();
        if (own != 0 && target >= in_front_of[t] && target < in_front_of[t] + own) {
          c.tokens[n] = (int)(uint32_t)mine[0];
          if (c.logprobs) c.logprobs[n] = (float)(((double)x - (double)r.top) * inv - log((double)sum / unit));
        }
        return;
      }
    } else if (!listed) {
      auto total_of = [&]() {
        unsigned long long sum = 0;
        each_token(row, 0, c.vocab, threadIdx.x, kThreads, [&](float x, int i) { sum += keeps(r, x, i) ? all(x) : 0ull; });
        sum = sum_over_wave(sum);
        __syncthreads();
        if (lane == 0) sm.sums[wave] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kWaves; ++w) sum += sm.sums[w];
        __syncthreads();
        return sum;
      };
      if (s.top_k > 0) cut(sm, row, c.vocab, r, all, false, s.top_k);
      if (s.top_p < 1.) {
        const unsigned long long total = total_of();
        const unsigned long long share = whole_share(s.top_p, (double)total), target = share < total ? share : total;
        cut(sm, row, c.vocab, r, all, true, target > 0 ? target : 1);
      }
    }
  }
  if (!listed) {
    unsigned long long sum = 0;
    each_token(row, 0, c.vocab, threadIdx.x, kThreads, [&](float x, int i) { sum += kept_weight(x, i); });
    sum = sum_over_wave(sum);
    __syncthreads();
    if (lane == 0) sm.sums[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kWaves; ++w) sum += sm.sums[w];
    __syncthreads();
    write(place_of<kThreads>(sm.place, row, 0, c.vocab, __umul64hi(sum, u64), kept_weight), (double)sum);
    return;
  }
  // what is kept of every part: what is above the list, and of the list
  unsigned long long* of_part = sm.mass;
  __syncthreads();
  for (int p = threadIdx.x; p < (space.n_parts + 63) / 64 * 64; p += kThreads) of_part[p] = p < space.n_parts ? parts[p].above : 0;
  __syncthreads();
  unsigned long long* of_sum = sm.place.sums;
  if (threadIdx.x < kSums) of_sum[threadIdx.x] = 0;
  unsigned long long kept_here[kList / kThreads] = {};
  if (s.cut()) {
#pragma unroll
    for (int q = 0; q < kList / kThreads; ++q) {
      const int j = q * kThreads + threadIdx.x;
      if (j >= cut_of_row.listed) continue;
      const unsigned long long e = listed_here[q];
      const uint32_t key = ~(uint32_t)(e >> 32);
      kept_here[q] = kept_weight(__uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key), (int)(uint32_t)e);
      if (kept_here[q]) atomicAdd(&of_part[(uint32_t)e / kPart], kept_here[q]);
    }
  }
  __syncthreads();
  // (every wavefront for itself)
  unsigned long long total = 0;
  for (int p = lane; p < space.n_parts; p += 64) total += of_part[p];
  total = sum_over_wave(total);
  unsigned long long way = __umul64hi(total, u64);
  int found = 0;
  for (int p0 = 0; p0 < space.n_parts; p0 += 64) {
    const unsigned long long own = of_part[p0 + lane];
    unsigned long long upto = own;
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned long long other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    const unsigned long long past = __ballot(way < upto);
    if (past) {
      const int at = __builtin_ctzll(past);
      found = p0 + at;
      way -= __shfl(upto - own, at);
      break;
    }
    way -= __shfl(upto, 63);
  }
  // the same in the part, whose sums the launch in front left, too
#pragma unroll
  for (int q = 0; q < kList / kThreads; ++q)
    if (kept_here[q] && (int)((uint32_t)listed_here[q] / kPart) == found) atomicAdd(&of_sum[(uint32_t)listed_here[q] % kPart / (kPart / kSums)], kept_here[q]);
  unsigned long long upto = lane < kSums && !list_is_all ? space.sums[((int64_t)blockIdx.x * space.n_parts + found) * kSums + lane] : 0;
  __syncthreads();
  if (lane < kSums) upto += of_sum[lane];
  const unsigned long long own = upto;
  for (int d = 1; d < kSums; d <<= 1) {
    const unsigned long long other = __shfl_up(upto, d);
    if (lane >= d) upto += other;
  }
  const int at = __builtin_ctzll(__ballot(lane < kSums && way < upto) | 1ull << (kSums - 1));
  way -= __shfl(upto - own, at);
  const int lo = found * kPart + at * (kPart / kSums);
  __syncthreads();
  write(place_of<kThreads>(sm.place, row, lo, min(lo + kPart / kSums, c.vocab), way, kept_weight), (double)total);
}

Space space_of(const SampleCall& c, int64_t rows) {
  Space s;
  s.n_parts = (c.vocab + kPart - 1) / kPart;                    // (at most kBins: vocab <= 2^24)
  s.rows = static_cast<RowSpace*>(c.workspace);
  const int64_t held = rows < kRowsAtOnce ? rows : kRowsAtOnce;
  s.parts = reinterpret_cast<Part*>(s.rows + held);
  s.sums = reinterpret_cast<unsigned long long*>(s.parts + held * s.n_parts);
  s.tops = reinterpret_cast<float*>(s.sums + held * s.n_parts * kSums);
  s.first_row = 0;
  return s;
}

template <typename T>
hipError_t launch_typed(const SampleCall& c, hipStream_t stream) {
  Space s = space_of(c, c.rows);
  const int bits = bits_of(c.vocab);
  // (what is given one a row may be anything)
  const bool cuts = c.top_ks || c.top_ps || (c.top_k > 0 && c.top_k < c.vocab) || c.top_p < 1., filters = cuts || c.min_ps || c.min_p > 0.;
  for (; s.first_row < c.rows; s.first_row += kRowsAtOnce) {
    const int64_t left = c.rows - s.first_row;
    const dim3 grid((unsigned)s.n_parts, (unsigned)(left < kRowsAtOnce ? left : kRowsAtOnce));
    // (eight tokens a thread where latency counts, 32 where there is enough to do)
    if ((int64_t)grid.x * grid.y < 1024) parts_kernel<T, kThreads><<<grid, kThreads, 0, stream>>>(c, s, bits, cuts);
    else parts_kernel<T, kFewThreads><<<grid, kFewThreads, 0, stream>>>(c, s, bits, cuts);
    if (cuts) bins_kernel<T><<<grid, kThreads, 0, stream>>>(c, s, bits);
    if (filters) collect_kernel<T><<<grid, kThreads, 0, stream>>>(c, s, bits);
    if (!filters && !c.temperatures && c.temperature > 0.) draw_plain_kernel<T><<<grid.y, kFewThreads, 0, stream>>>(c, s, bits);
    else draw_kernel<T><<<grid.y, kThreads, 0, stream>>>(c, s, bits);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace

size_t sample_workspace(int rows, int vocab) {
  SampleCall c = {};
  c.vocab = vocab;
  const Space s = space_of(c, rows);
  return (size_t)(rows < kRowsAtOnce ? rows : kRowsAtOnce) * (sizeof(RowSpace) + (size_t)s.n_parts * (sizeof(Part) + kSums * sizeof(unsigned long long) + kChunks * sizeof(float)));
}

hipError_t launch_sample(const SampleCall& c, int dtype, hipStream_t stream) {
  return dtype == RLKV_F32 ? launch_typed<float>(c, stream) : launch_typed<uint16_t>(c, stream);
}

}  // namespace rlkv
