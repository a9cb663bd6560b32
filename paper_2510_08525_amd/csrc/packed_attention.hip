// Attention over whole sequences packed one behind the other, causal or local (sinks and recent positions):
//
//   out[i] = sum_j w[i][j] v[j] / sum_j w[i][j],   w[i][j] = exp(scale q[i] . k[j]),   j admitted to i;   lse[i] = log sum_j w[i][j]
//
// A workgroup has 256 columns (packed_attention.h) of one KV head, 32 a wavefront, and walks once over the keys that any of them
// admits, 64 at a time, with the running maximum and sum of each column: its first position's sequence begins where the keys begin, and the
// few keys of other sequences are masked.  So blocks of columns need no plan, sequences of any lengths (none among them) fill them, and the launch is
// the same whatever the offsets hold.  Keys x queries first: scores, weights, maximum and sum of a column are in its two lanes.
#include "packed_attention.h"

namespace rlkv {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kKeys = 64, kColumns = 32 * kWaves;
constexpr int kUnits = kKeys * 16 / kThreads;       // 16-byte units of a tile that a thread brings

struct Smem {
  uint4 k[2][kKeys * 16], v[2][kKeys * 16];
  int32_t offsets[kOffsetsInLds];
  int32_t first[kWaves], begin[kWaves], last[kWaves];
};

__global__ __launch_bounds__(kThreads) void packed_attention_kernel(PackedCall c) {
  __shared__ Smem sm;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int h = blockIdx.y, group = c.group;
  const bool full = (c.full[h >> 6] >> (h & 63)) & 1;

  // the column of the lane, its position, and where its sequence begins
  const int32_t* offsets = c.offsets;
  if (c.n_seqs < kOffsetsInLds) {
    for (int i = threadIdx.x; i <= c.n_seqs; i += kThreads) sm.offsets[i] = c.offsets[i];
    __syncthreads();
    offsets = sm.offsets;
  }
  const int64_t column = (int64_t)blockIdx.x * kColumns + wave * 32 + (lane & 31);
  int pos = (int)(column / group);
  const int head = h * group + (int)(column - (int64_t)pos * group);
  const Span span = span_of(offsets, c.n_seqs, c.tokens, pos);
  const bool valid = span.begin >= 0;
  const int begin = valid ? span.begin : 0;
  const int64_t row = valid ? pos : 0;                       // (a column of no sequence reads row 0 and writes nothing)
  // of the wavefront: first and last position, first and last beginning
  const int pos_lo = min_of_lanes(valid ? pos : INT32_MAX), pos_hi = max_of_lanes(valid ? pos : -1);
  const int begin_lo = min_of_lanes(valid ? begin : INT32_MAX), begin_hi = max_of_lanes(valid ? begin : -1);
  if (lane == 0) {
    sm.first[wave] = pos_lo;
    sm.begin[wave] = begin_lo;
    sm.last[wave] = pos_hi;
  }
  __syncthreads();
  int first = INT32_MAX, keys_begin = INT32_MAX, last = -1;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    first = min(first, sm.first[w]);
    keys_begin = min(keys_begin, sm.begin[w]);
    last = max(last, sm.last[w]);
  }
  if (last < 0) return;

  bf16x8 q[8];
  const uint16_t* q_row = c.q.p + row * c.q.token + head * c.q.head + 8 * half;
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q_row + 16 * s));

  // Tiles: of a full head from keys_begin on; of a local one those of the sinks of the first sequence, then from the first position's band on
  // (later sequences of the block begin behind the first position).
  const int sink_tiles = full ? 0 : (int)(((int64_t)min(c.sink, last + 1 - keys_begin) + kKeys - 1) / kKeys);
  const int band = full ? keys_begin : max(keys_begin + sink_tiles * kKeys, first - c.recent + 1);
  const int tiles = sink_tiles + (band > last ? 0 : (last - band) / kKeys + 1);
  auto tile_key = [&](int t) { return t < sink_tiles ? keys_begin + t * kKeys : band + (t - sink_tiles) * kKeys; };

  uint4 next_k[kUnits], next_v[kUnits];
  auto fetch = [&](int t) {
    const int k0 = tile_key(t);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int at = threadIdx.x + i * kThreads, r = min(k0 + (at >> 4), c.tokens - 1), u = at & 15;
      next_k[i] = *reinterpret_cast<const uint4*>(c.k.p + (int64_t)r * c.k.token + h * c.k.head + u * 8);
      next_v[i] = *reinterpret_cast<const uint4*>(c.v.p + (int64_t)r * c.v.token + h * c.v.head + u * 8);
    }
  };
  auto place = [&](int slot) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int at = threadIdx.x + i * kThreads;
      sm.k[slot][unit_at(at >> 4, at & 15)] = next_k[i];
      sm.v[slot][unit_at(at >> 4, at & 15)] = next_v[i];
    }
  };

  const float scale = c.scale * kLog2e;
  auto admits = [&](int key) { return key <= pos && key >= begin && (full || key - begin < c.sink || pos - key < c.recent); };

  // A weight of 0 does not keep an infinity or a NaN of a masked value out of the products.  Where an output is not finite, the whole walk is taken
  // again with the products of masked tiles one by one (careful).
  floatx16 o[4];
  float m, l;
  for (int careful = 0;; careful = 1) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    fetch(0);
    place(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
      const int slot = t & 1, k0 = tile_key(t), k1 = k0 + kKeys - 1;
      if (t + 1 < tiles) fetch(t + 1);
      const bool some = k0 <= pos_hi && k1 >= begin_lo && (full || k0 - begin_hi < c.sink || pos_lo - k1 < c.recent);
      if (some) {
        const bool all = k1 <= pos_lo && k0 >= begin_hi && (full || k1 - begin_lo < c.sink || pos_hi - k0 < c.recent);
        floatx16 x[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int r = 0; r < 16; ++r) x[b][r] = 0.f;
#pragma unroll
          for (int s = 0; s < 8; ++s)
            x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment(sm.k[slot], 32 * b, s), q[s], x[b], 0, 0, 0);
        }
        if (!all) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (!admits(k0 + 32 * b + 8 * (r >> 2) + 4 * half + (r & 3))) x[b][r] = -INFINITY;
        }
        float mx = m;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[b][r]);
        mx = max_of_halves(mx);
        const float ref = mx == -INFINITY ? 0.f : mx * scale;
        const float alpha = __builtin_amdgcn_exp2f(m * scale - ref);
        m = mx;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[b][r] *= alpha;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            x[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r], scale, -ref));
            l += x[b][r];
          }
        if (careful && !all) {
          for (int key = 0; key < kKeys; ++key) {
            float w = 0.f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (32 * b + 8 * (r >> 2) + (r & 3) == (key & ~4)) w = x[b][r];
            const float other = other_half(w);
            if (((key >> 2) & 1) != half) w = other;
            if (!admits(k0 + key)) continue;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const int d = 32 * b + 8 * g + 4 * half;
                const words2 two = *reinterpret_cast<const words2*>(reinterpret_cast<const char*>(&sm.v[slot][unit_at(key, d >> 3)]) + 2 * (d & 7));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[b][4 * g + e] += w * __uint_as_float(e & 1 ? two[e >> 1] & 0xffff0000u : two[e >> 1] << 16);
              }
          }
        } else {
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const bf16x8 w = weights_fragment(x[s >> 1], s & 1);
#pragma unroll
            for (int b = 0; b < 4; ++b)
              o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment(sm.v[slot], 16 * s, b), w, o[b], 0, 0, 0);
          }
        }
      }
      if (t + 1 < tiles) place(slot ^ 1);
      __syncthreads();
    }
    if (careful) break;
    float all = 0.f;                                          // (x * 0 is 0 or NaN)
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) all += o[b][r] * 0.f;
    if (!__syncthreads_or(valid && all != 0.f)) break;
  }

  l = sum_of_halves(l);
  if (!valid) return;
  const float inv = 1.f / l;
  uint16_t* out = c.out.p + row * c.out.token + head * c.out.head;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const words2 w = {two_bf16(o[b][4 * g] * inv, o[b][4 * g + 1] * inv), two_bf16(o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv)};
      *reinterpret_cast<words2*>(out + 32 * b + 8 * g + 4 * half) = w;
    }
  if (c.lse && half == 0) c.lse[(int64_t)head * c.tokens + pos] = m * c.scale + logf(l);
}

}  // namespace

hipError_t launch_packed_attention(const PackedCall& call, hipStream_t stream) {
  const int64_t columns = (int64_t)call.tokens * call.group;
  const dim3 grid((uint32_t)((columns + kColumns - 1) / kColumns), (uint32_t)call.n_kv_heads);
  packed_attention_kernel<<<grid, kThreads, 0, stream>>>(call);
  return hipGetLastError();
}

}  // namespace rlkv
