// Attention over whole sequences packed one behind the other, causal or local (sinks and recent positions):
//
//   out[i] = sum_j w[i][j] v[j] / sum_j w[i][j],   w[i][j] = exp(scale q[i] . k[j]),   j admitted to i;   lse[i] = log sum_j w[i][j]
//
// A workgroup has 256 columns (packed_attention.h) of one KV head, 32 a wavefront, and walks once over the keys that any of them
// admits, 64 at a time, with the running maximum and sum of each column: its first position's sequence begins where the keys begin, and the
// few keys of other sequences are masked.  So blocks of columns need no plan, sequences of any lengths (none among them) fill them, and the launch is
// the same whatever the offsets hold.  Keys x queries first: scores, weights, maximum and sum of a column are in its two lanes.
//
// 4 * 128 operations a pair of an admitted key and a query head.  One sequence of 16384 tokens, 32 / 8 heads: 1990 us (1890 to 2085 over machines), 1.11 PFLOP/s
// where the library's product of 8192^3 reaches 1.23: the matrix cores are busy for 57 % of the time, and in the rest of it the vector instructions are, some 180 a
// wavefront and tile (exponentials, maxima, rounding), with which they hardly overlap; reads of LDS (128 bytes a clock) take less.  24 sequences of 100
// to 2000 tokens, 28 / 4 heads, half of them local: 251 to 272 us, of which each of the eleven workgroups that a compute unit has one after the other spends 9 on
// its start and end (offsets, queries, the first tile, the stores): with 256 registers a lane there is no second one beside it.
#include "packed_attention.h"

namespace rlkv {
namespace {

// The reference of the weights moves only when a score is more than this above it (in powers of two): until then weights are above 1, which costs
// fp32 sums and bf16 weights nothing, and the accumulators stay as they are.
constexpr float kSlack = 8.f;
// A reference is a product rounded to fp32, while the products that it is taken from are not (one rounding for the difference): the largest weight is off 1
// by up to half a step of the reference, 2^2 from here on, 2^64 at 2^31, and fits no float beyond.  From here on the walk is taken again with the
// products' differences taken before the scale (careful), which the rounding of neither product enters.  (333 tokens, 28 / 4 heads: 55 us for 13, most of it the
// masked tiles' products one by one.)
constexpr float kLargeReference = 67108864.f;          // 2^26

// SPLIT 2: the keys are divided between the halves of the workgroup (keys_divided).
template <int WAVES, int SPLIT>
__global__ __launch_bounds__(64 * WAVES) void packed_attention_kernel(PackedCall c, uint32_t blocks) {
  constexpr int kColumnWaves = WAVES / SPLIT;
  // (objects of their own, and the buffer of a tile known at compile time: else reads of one tile would wait for the loads of the next)
  __shared__ uint4 t0[SPLIT][2][kKeys * 16], t1[SPLIT][2][kKeys * 16];      // keys, values
  __shared__ int32_t lost;
  const int half = (threadIdx.x >> 5) & 1, part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kColumnWaves : 0;
  const Offsets offsets(c);
  const ColumnBlock block = column_block(c, blockIdx.x, blocks);
  Columns x;
  if (!set_columns<kColumnWaves>(c, offsets, block, x)) return;
  if (threadIdx.x == 0) lost = 0;

  bf16x8 q[8];
  {
    const uint16_t* row = c.q.p + x.row * c.q.token + x.head * c.q.head + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + 16 * s));
  }
  const float scale = c.scale * kLog2e, slack = kSlack / scale;
  auto ask = [&](auto odd, int t) {
    constexpr int kOdd = decltype(odd)::value;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i) {
      if (i > 0 && t + i >= x.tiles) break;
      stage_rows<kPairs, WAVES>(c.k, x.tile_key(t + i), block.head, c.tokens, kOdd ? t1[i][0] : t0[i][0]);
      stage_rows<kPairs, WAVES>(c.v, x.tile_key(t + i), block.head, c.tokens, kOdd ? t1[i][1] : t0[i][1]);
    }
  };

  floatx16 o[4];
  float m, l, ref;
  // A weight of 0 does not keep an infinity or a NaN of a masked value out of the products.  Where an output is not finite, the walk is taken again
  // with the products of masked tiles one by one (careful), and where references are large.
  auto walk = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
    m = -INFINITY;
    l = ref = 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) clear(o[b]);
    ask(std::integral_constant<int, 0>{}, 0);
    auto step = [&](auto odd, int t) {
      constexpr int kOdd = decltype(odd)::value;
      const uint4 *kt = kOdd ? t1[part][0] : t0[part][0], *vt = kOdd ? t1[part][1] : t0[part][1];
      tile_arrived();
      if (t + SPLIT < x.tiles) ask(std::integral_constant<int, 1 - kOdd>{}, t + SPLIT);
      if (part > 0 && t + part >= x.tiles) return;
      const int key = x.tile_key(t + part);
      if (!x.any_of(key, kKeys)) return;
      const bool all = x.all_of(key, kKeys);
      floatx16 w[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) clear(w[b]);
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int b = 0; b < 2; ++b) w[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment<kPairs>(kt, 32 * b, s), q[s], w[b], 0, 0, 0);
      reads_ahead<16, 16, 6, 1>();
      if (!all) {
        x.mask(w[0], key, -INFINITY);
        x.mask(w[1], key + 32, -INFINITY);
      }
      float mx = fmaxf(w[0][0], w[1][0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(fmaxf(mx, w[0][r]), w[1][r]);
      if (__any(mx > m + slack)) {
        mx = fmaxf(max_of_halves(mx), m);
        const float next = mx == -INFINITY ? 0.f : mx * scale;
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(kCareful ? (m - mx) * scale : ref - next);
        m = mx;
        ref = next;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < 4; ++b) o[b] *= alpha;
      }
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          w[b][r] = __builtin_amdgcn_exp2f(kCareful ? (w[b][r] - from) * scale : __builtin_fmaf(w[b][r], scale, -ref));
          l += w[b][r];
        }
      if (kCareful && !all) {
#pragma unroll
        for (int b = 0; b < 2; ++b) admitted_products<kPairs>(vt, 32 * b, w[b], o, [&](int r) { return x.admits(key + 32 * b + r); });
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const bf16x8 p = weights_fragment(w[s >> 1], s & 1);
#pragma unroll
          for (int b = 0; b < 4; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment<kPairs>(vt, 16 * s, b), p, o[b], 0, 0, 0);
        }
        reads_ahead<16, 32, 8, 2>();
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
  const bool again = any_of_workgroup(x.valid && (zero_or_nan(o) + l * 0.f != 0.f || fabsf(ref) >= kLargeReference), lost);
  if (again) walk(std::true_type{});

  l = sum_of_halves(l);
  if (SPLIT > 1) {
    // the second half's sums to the first: by lanes, piece behind piece, in the tiles' place
    float4* sums = reinterpret_cast<float4*>(t0);
    float4* stats = reinterpret_cast<float4*>(t1);
    const int at = threadIdx.x % (64 * kColumnWaves);
    __syncthreads();
    if (part == 1) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        sums[i * 64 * kColumnWaves + at] = make_float4(o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]);
      stats[at] = make_float4(m, l, ref, 0.f);
    }
    __syncthreads();
    if (part == 1) return;
    // (from reference to reference as the weights have them: the products of m would be taken unrounded into the differences, and from scores of some
    // ten thousand on the halves' weights would not fit each other)
    const float4 other = stats[at];
    const float most = fmaxf(m, other.x), next = m < other.x ? other.z : ref;
    const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(again ? (m - most) * scale : ref - next);
    const float its = other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(again ? (other.x - most) * scale : other.z - next);
    m = most;
    l = l * mine + other.y * its;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float4 y = sums[i * 64 * kColumnWaves + at];
      o[i >> 2][4 * (i & 3)] = o[i >> 2][4 * (i & 3)] * mine + y.x * its;
      o[i >> 2][4 * (i & 3) + 1] = o[i >> 2][4 * (i & 3) + 1] * mine + y.y * its;
      o[i >> 2][4 * (i & 3) + 2] = o[i >> 2][4 * (i & 3) + 2] * mine + y.z * its;
      o[i >> 2][4 * (i & 3) + 3] = o[i >> 2][4 * (i & 3) + 3] * mine + y.w * its;
    }
  }
  store_rows(c.out.p + x.row * c.out.token + x.head * c.out.head, o, __builtin_amdgcn_rcpf(l), x.valid);
  if (c.lse && x.valid && half == 0) c.lse[(int64_t)x.head * c.tokens + x.pos] = m * c.scale + __builtin_amdgcn_logf(l) * kLn2;
}

}  // namespace

hipError_t launch_packed_attention(const PackedCall& call, hipStream_t stream) {
  const uint32_t blocks = column_blocks(call, kPackedWaves), few = column_blocks(call, kPackedWaves / 2);
  if (keys_divided(call))
    packed_attention_kernel<kPackedWaves, 2><<<few * (uint32_t)call.n_kv_heads, 64 * kPackedWaves, 0, stream>>>(call, few);
  else
    packed_attention_kernel<kPackedWaves, 1><<<blocks * (uint32_t)call.n_kv_heads, 64 * kPackedWaves, 0, stream>>>(call, blocks);
  return hipGetLastError();
}

}  // namespace rlkv
