// Gradient of the packed attention (packed_attention.hip).  With w[i][j] = exp(scale q[i] . k[j] - lse[i]) of the admitted pairs:
//
//   delta[i] = grad_out[i] . out[i]          z[i][j] = w[i][j] (grad_out[i] . v[j] - delta[i])
//   grad_q[i] = scale sum_j z[i][j] k[j]     grad_k[j] = scale sum_i z[i][j] q[i]     grad_v[j] = sum_i w[i][j] grad_out[i]
//
// Two kernels, each of which forms w and z for itself: one walks over the keys of its columns (queries) as the forward one does and leaves grad_q
// and delta, the other over the columns of its keys and leaves grad_k and grad_v, summed over the group's heads in fp32 in a fixed order.
// That is seven products where one kernel would do five, but none of them adds to memory that others add to: equal calls give equal bits.
#include "packed_attention.h"

namespace rlkv {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

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
// Result [d][column] as a row of the column's lanes.
__device__ __forceinline__ void store_rows(uint16_t* row, const floatx16 (&x)[4], float scale) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const words2 w = {two_bf16(x[b][4 * g] * scale, x[b][4 * g + 1] * scale), two_bf16(x[b][4 * g + 2] * scale, x[b][4 * g + 3] * scale)};
      *reinterpret_cast<words2*>(row + 32 * b + 8 * g + 4 * half) = w;
    }
}
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

// ---- queries ------------------------------------------------------------------------------------------------------------------
constexpr int kColumns = 32 * kWaves, kKeys = 64;
constexpr int kKeyUnits = kKeys * 16 / kThreads;

struct QuerySmem {
  uint4 k[2][kKeys * 16], v[2][kKeys * 16];
  int32_t offsets[kOffsetsInLds];
  int32_t first[kWaves], begin[kWaves], last[kWaves];
};

__global__ __launch_bounds__(kThreads) void packed_grad_q_kernel(PackedCall c) {
  __shared__ QuerySmem sm;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int h = blockIdx.y, group = c.group;
  const bool full = (c.full[h >> 6] >> (h & 63)) & 1;
  const int32_t* offsets = c.offsets;
  if (c.n_seqs < kOffsetsInLds) {
    for (int i = threadIdx.x; i <= c.n_seqs; i += kThreads) sm.offsets[i] = c.offsets[i];
    __syncthreads();
    offsets = sm.offsets;
  }
  const int64_t column = (int64_t)blockIdx.x * kColumns + wave * 32 + (lane & 31);
  const int pos = (int)(column / group);
  const int head = h * group + (int)(column - (int64_t)pos * group);
  const Span span = span_of(offsets, c.n_seqs, c.tokens, pos);
  const bool valid = span.begin >= 0;
  const int begin = valid ? span.begin : 0;
  const int64_t row = valid ? pos : 0;
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

  bf16x8 q[8], g[8];
  float delta = 0.f;
  const uint16_t* q_row = c.q.p + row * c.q.token + head * c.q.head + 8 * half;
  const uint16_t* g_row = c.grad_out.p + row * c.grad_out.token + head * c.grad_out.head + 8 * half;
  const uint16_t* o_row = c.out.p + row * c.out.token + head * c.out.head + 8 * half;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q_row + 16 * s));
    const uint4 gw = *reinterpret_cast<const uint4*>(g_row + 16 * s);
    g[s] = __builtin_bit_cast(bf16x8, gw);
    delta += dot_of_units(gw, *reinterpret_cast<const uint4*>(o_row + 16 * s));
  }
  delta = sum_of_halves(delta);
  const float lse = valid ? c.lse[(int64_t)head * c.tokens + pos] * kLog2e : 0.f;
  if (valid && half == 0) c.delta[(int64_t)head * c.tokens + pos] = delta;

  const int sink_tiles = full ? 0 : (int)(((int64_t)min(c.sink, last + 1 - keys_begin) + kKeys - 1) / kKeys);
  const int band = full ? keys_begin : max(keys_begin + sink_tiles * kKeys, first - c.recent + 1);
  const int tiles = sink_tiles + (band > last ? 0 : (last - band) / kKeys + 1);
  auto tile_key = [&](int t) { return t < sink_tiles ? keys_begin + t * kKeys : band + (t - sink_tiles) * kKeys; };

  uint4 next_k[kKeyUnits], next_v[kKeyUnits];
  auto fetch = [&](int t) {
    const int k0 = tile_key(t);
#pragma unroll
    for (int i = 0; i < kKeyUnits; ++i) {
      const int at = threadIdx.x + i * kThreads, r = min(k0 + (at >> 4), c.tokens - 1), u = at & 15;
      next_k[i] = *reinterpret_cast<const uint4*>(c.k.p + (int64_t)r * c.k.token + h * c.k.head + u * 8);
      next_v[i] = *reinterpret_cast<const uint4*>(c.v.p + (int64_t)r * c.v.token + h * c.v.head + u * 8);
    }
  };
  auto place = [&](int slot) {
#pragma unroll
    for (int i = 0; i < kKeyUnits; ++i) {
      const int at = threadIdx.x + i * kThreads;
      sm.k[slot][unit_at(at >> 4, at & 15)] = next_k[i];
      sm.v[slot][unit_at(at >> 4, at & 15)] = next_v[i];
    }
  };
  const float scale = c.scale * kLog2e;
  auto admits = [&](int key) { return key <= pos && key >= begin && (full || key - begin < c.sink || pos - key < c.recent); };

  floatx16 dq[4];
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int b = 0; b < 4; ++b) clear(dq[b]);
    fetch(0);
    place(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
      const int slot = t & 1, k0 = tile_key(t), k1 = k0 + kKeys - 1;
      if (t + 1 < tiles) fetch(t + 1);
      const bool some = k0 <= pos_hi && k1 >= begin_lo && (full || k0 - begin_hi < c.sink || pos_lo - k1 < c.recent);
      if (some) {
        const bool all = k1 <= pos_lo && k0 >= begin_hi && (full || k1 - begin_lo < c.sink || pos_hi - k0 < c.recent);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          floatx16 x, y;
          clear(x);
          clear(y);
#pragma unroll
          for (int s = 0; s < 8; ++s) {
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment(sm.k[slot], 32 * b, s), q[s], x, 0, 0, 0);
            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment(sm.v[slot], 32 * b, s), g[s], y, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], scale, -lse)) * (y[r] - delta);
          if (!all) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (!admits(k0 + 32 * b + 8 * (r >> 2) + 4 * half + (r & 3))) x[r] = 0.f;
          }
          if (careful && !all) {
            admitted_products(sm.k[slot], 32 * b, x, dq, [&](int r) { return admits(k0 + 32 * b + r); });
          } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const bf16x8 z = weights_fragment(x, s);
#pragma unroll
              for (int d = 0; d < 4; ++d)
                dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment(sm.k[slot], 32 * b + 16 * s, d), z, dq[d], 0, 0, 0);
            }
          }
        }
      }
      if (t + 1 < tiles) place(slot ^ 1);
      __syncthreads();
    }
    if (careful || !__syncthreads_or(valid && zero_or_nan(dq) != 0.f)) break;
  }
  if (valid) store_rows(c.grad_q.p + row * c.grad_q.token + head * c.grad_q.head, dq, c.scale);
}

// ---- keys and values ----------------------------------------------------------------------------------------------------------
// A workgroup has 256 keys, 32 a wavefront and one a lane (both halves of the wavefront: the same), and walks over the columns that admit any of
// them, 32 at a time.  Key j is admitted to the positions j <= i < limit: the end of its sequence, or of a local head's key that is no sink
// j + recent if that is less.
constexpr int kKeysHere = 32 * kWaves, kStep = 32;

struct KeySmem {
  uint4 q[2][kStep * 16], g[2][kStep * 16];
  float lse[2][kStep], delta[2][kStep];
  int32_t pos[2][kStep];
  int32_t offsets[kOffsetsInLds];
  int32_t first[kWaves], limit[kWaves];
};

__global__ __launch_bounds__(kThreads) void packed_grad_kv_kernel(PackedCall c) {
  __shared__ KeySmem sm;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int h = blockIdx.y, group = c.group;
  const bool full = (c.full[h >> 6] >> (h & 63)) & 1;
  const int32_t* offsets = c.offsets;
  if (c.n_seqs < kOffsetsInLds) {
    for (int i = threadIdx.x; i <= c.n_seqs; i += kThreads) sm.offsets[i] = c.offsets[i];
    __syncthreads();
    offsets = sm.offsets;
  }
  const int key = blockIdx.x * kKeysHere + wave * 32 + (lane & 31);
  const Span span = span_of(offsets, c.n_seqs, c.tokens, key);
  const bool valid = span.begin >= 0;
  const int64_t row = valid ? key : 0;
  const int limit = !valid ? -1 : full || key - span.begin < c.sink || span.end - key < c.recent ? span.end : key + c.recent;
  const int key_lo = min_of_lanes(valid ? key : INT32_MAX), key_hi = max_of_lanes(valid ? key : -1);
  const int limit_lo = min_of_lanes(valid ? limit : INT32_MAX), limit_hi = max_of_lanes(limit);
  if (lane == 0) {
    sm.first[wave] = key_lo;
    sm.limit[wave] = limit_hi;
  }
  __syncthreads();
  int first = INT32_MAX, end = -1;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    first = min(first, sm.first[w]);
    end = max(end, sm.limit[w]);
  }
  if (end < 0) return;

  bf16x8 k[8], v[8];
  const uint16_t* k_row = c.k.p + row * c.k.token + h * c.k.head + 8 * half;
  const uint16_t* v_row = c.v.p + row * c.v.token + h * c.v.head + 8 * half;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    k[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(k_row + 16 * s));
    v[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(v_row + 16 * s));
  }

  // Columns past the last one are given position -1, which admits no key, and the row of the last one.
  const int64_t column0 = (int64_t)first * group, column_end = (int64_t)end * group;
  const int steps = (int)((column_end - column0 + kStep - 1) / kStep);
  uint4 next_q, next_g;
  float next_lse = 0.f, next_delta = 0.f;
  int next_pos = -1;
  auto fetch = [&](int t) {
    const int r = threadIdx.x >> 4, u = threadIdx.x & 15;
    const int64_t col = column0 + (int64_t)t * kStep + r, at = col < column_end ? col : column_end - 1;
    const int p = (int)(at / group), head = h * group + (int)(at - (int64_t)p * group);
    next_q = *reinterpret_cast<const uint4*>(c.q.p + (int64_t)p * c.q.token + head * c.q.head + u * 8);
    next_g = *reinterpret_cast<const uint4*>(c.grad_out.p + (int64_t)p * c.grad_out.token + head * c.grad_out.head + u * 8);
    if (u == 0) {
      next_lse = c.lse[(int64_t)head * c.tokens + p] * kLog2e;
      next_delta = c.delta[(int64_t)head * c.tokens + p];
      next_pos = col < column_end ? p : -1;
    }
  };
  auto place = [&](int slot) {
    const int r = threadIdx.x >> 4, u = threadIdx.x & 15;
    sm.q[slot][unit_at(r, u)] = next_q;
    sm.g[slot][unit_at(r, u)] = next_g;
    if (u == 0) {
      sm.lse[slot][r] = next_lse;
      sm.delta[slot][r] = next_delta;
      sm.pos[slot][r] = next_pos;
    }
  };
  const float scale = c.scale * kLog2e;

  floatx16 dk[4], dv[4];
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      clear(dk[b]);
      clear(dv[b]);
    }
    fetch(0);
    place(0);
    __syncthreads();
    for (int t = 0; t < steps; ++t) {
      const int slot = t & 1;
      if (t + 1 < steps) fetch(t + 1);
      const int64_t c0 = column0 + (int64_t)t * kStep, c1 = c0 + kStep - 1;
      const int pos_lo = (int)(c0 / group), pos_hi = (int)((c1 < column_end ? c1 : column_end - 1) / group);
      if (pos_hi >= key_lo && pos_lo < limit_hi) {
        const bool all = c1 < column_end && pos_lo >= key_hi && pos_hi < limit_lo;
        floatx16 x, y;
        clear(x);
        clear(y);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment(sm.q[slot], 0, s), k[s], x, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_fragment(sm.g[slot], 0, s), v[s], y, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int col = 8 * (r >> 2) + 4 * half + (r & 3);
          x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], scale, -sm.lse[slot][col]));
          y[r] = x[r] * (y[r] - sm.delta[slot][col]);
        }
        auto admits = [&](int col) { return valid && sm.pos[slot][col] >= key && sm.pos[slot][col] < limit; };
        if (!all) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!admits(8 * (r >> 2) + 4 * half + (r & 3))) x[r] = y[r] = 0.f;
        }
        if (careful && !all) {
          admitted_products(sm.g[slot], 0, x, dv, admits);
          admitted_products(sm.q[slot], 0, y, dk, admits);
        } else {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const bf16x8 w = weights_fragment(x, s), z = weights_fragment(y, s);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment(sm.g[slot], 16 * s, d), w, dv[d], 0, 0, 0);
              dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_fragment(sm.q[slot], 16 * s, d), z, dk[d], 0, 0, 0);
            }
          }
        }
      }
      if (t + 1 < steps) place(slot ^ 1);
      __syncthreads();
    }
    if (careful || !__syncthreads_or(valid && (zero_or_nan(dk) != 0.f || zero_or_nan(dv) != 0.f))) break;
  }
  if (!valid) return;
  store_rows(c.grad_k.p + row * c.grad_k.token + h * c.grad_k.head, dk, c.scale);
  store_rows(c.grad_v.p + row * c.grad_v.token + h * c.grad_v.head, dv, 1.f);
}

}  // namespace

size_t packed_grad_workspace(int tokens, int n_q_heads, int) { return ((size_t)tokens * n_q_heads * sizeof(float) + 15) / 16 * 16; }

hipError_t launch_packed_attention_grad(PackedCall call, hipStream_t stream) {
  call.delta = static_cast<float*>(call.workspace);
  const int64_t columns = (int64_t)call.tokens * call.group;
  packed_grad_q_kernel<<<dim3((uint32_t)((columns + kColumns - 1) / kColumns), (uint32_t)call.n_kv_heads), kThreads, 0, stream>>>(call);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  packed_grad_kv_kernel<<<dim3((uint32_t)((call.tokens + kKeysHere - 1) / kKeysHere), (uint32_t)call.n_kv_heads), kThreads, 0, stream>>>(call);
  return hipGetLastError();
}

}  // namespace rlkv
