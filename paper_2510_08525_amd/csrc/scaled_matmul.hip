// Product of two 8-bit matrices whose scales change along the inner dimension:
//
//   out[m][n] = sum_g  sa[g][m] * sb[n / 128][g] * sum_{k in group g} a[m][k] * b[n][k]          (groups of 128 k)
//
// A group's partial product starts from zero and enters the fp32 sums by fused multiply-adds with the two scales' product: the
// scales cost vector instructions beside the matrix cores' time.  There are two ways to the partial product of a 16 x 16 tile:
//
//   kWide   the 8-bit values become 16-bit ones, exactly (4 instructions for 8 values of a lane), and four v_mfma_f32_16x16x32_f16 sum
//           their exact products in fp32
//   kFast   one v_mfma_f32_16x16x128_f8f6f4.  The sums inside that instruction are not fp32: it aligns the products of
//           neighbouring k to the largest of them and drops what lies more than 13 binary places below that product's exponent
//           (found with single products: -416 * 160 - 0.25 * 14 gives -66560).  Values within a factor of 2^7 of the group's largest
//           product lose nothing, and it has twice the rate and converts nothing.
//
// An fp32 output is always of the first kind, and so are few rows, where b's bytes are what counts; many rows with a bf16 output take the
// second.  b is the instruction's first operand:
// a lane's four results then belong to one row of a, whose scale is one register, and to four neighbouring columns of the output.  The order
// of k inside a group does not matter as long as both operands have the same: lane (row, seg) holds bytes [16 seg, 16 seg + 16) and the
// same 64 further on, so that a load of 16 lanes x 4 segments reads 64 contiguous bytes of each row.
#include <type_traits>

#include "token_ops.h"

namespace rlkv {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
#define RLKV_GLOBAL const __attribute__((address_space(1)))
#define RLKV_LDS __attribute__((address_space(3)))

typedef _Float16 halves2 __attribute__((ext_vector_type(2)));
typedef _Float16 halves8 __attribute__((ext_vector_type(8)));

enum { kWide, kFast };
template <int WAY> struct Operand;                     // a lane's 32 values of a group
template <> struct Operand<kFast> { i32x8 v; };
template <> struct Operand<kWide> { halves8 v[4]; };

__device__ __forceinline__ void to_operand(const i32x8& bytes, Operand<kFast>& o) { o.v = bytes; }
__device__ __forceinline__ void to_operand(const i32x8& bytes, Operand<kWide>& o) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const halves2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes[i], 1.f, false);
    const halves2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes[i], 1.f, true);
    halves8& to = o.v[i >> 1];
    const int at = (i & 1) * 4;
    to[at] = lo[0]; to[at + 1] = lo[1]; to[at + 2] = hi[0]; to[at + 3] = hi[1];
  }
#endif
}
__device__ __forceinline__ floats4 group_product(const Operand<kFast>& b, const Operand<kFast>& a) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, floats4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#else
  return floats4{};
#endif
}
__device__ __forceinline__ floats4 group_product(const Operand<kWide>& b, const Operand<kWide>& a) {
  floats4 p = {0.f, 0.f, 0.f, 0.f};
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.v[i], a.v[i], p, 0, 0, 0);
#endif
  return p;
}
__device__ __forceinline__ i32x8 both(const i32x4& lo, const i32x4& hi) {
  return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

__device__ __forceinline__ void store_four(const MatmulCall& c, int m, int n, const floats4& v, bool bf16) {
  if (m >= c.m || n >= c.n) return;
  if (bf16) {
    uint16_t* p = static_cast<uint16_t*>(c.out) + m * c.out_stride + n;
    const words2 w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    if (c.whole_out && n + 4 <= c.n) {
      *reinterpret_cast<words2*>(p) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < c.n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  } else {
    float* p = static_cast<float*>(c.out) + m * c.out_stride + n;
    if (c.whole_out && n + 4 <= c.n) {
      *reinterpret_cast<floats4*>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < c.n) p[i] = v[i];
    }
  }
}

// ---- few rows of a: b is read once, straight into registers -------------------------------------------------------------------
// A workgroup has 16 rows of b; its wavefronts take every eighth group of k and add their sums in LDS.  NT tiles of 16 rows of a.
constexpr int kFewWaves = 8;

template <int NT, bool BF16>
__global__ __launch_bounds__(kFewWaves * 64) void few_rows_kernel(MatmulCall c) {
  __shared__ floats4 parts[kFewWaves][NT][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, row = lane & 15, seg = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * NT * 16;
  constexpr int kFewAhead = NT < 4 ? 4 : 2;                        // groups whose loads are in flight together
  const int groups = (c.k + kGroup - 1) / kGroup;
  const int n_row = n0 + row < c.n ? n0 + row : c.n - 1;           // (rows past the end repeat the last one and are not stored)
  const char* b = static_cast<const char*>(c.b) + n_row * c.b_stride + seg * 16;
  const char* a[NT];
  int m_row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_row[t] = m0 + t * 16 + row < c.m ? m0 + t * 16 + row : c.m - 1;
    a[t] = static_cast<const char*>(c.a) + m_row[t] * c.a_stride + seg * 16;
  }
  const float* b_scales = c.b_scales + (n0 / kGroup) * c.b_scale_stride;
  floats4 acc[NT] = {};
  auto chunk = [&](const char* p, int k) {       // 16 bytes, zeros past the end of k
    i32x4 v = {0, 0, 0, 0};
    if (k + seg * 16 < c.k) v = *reinterpret_cast<const i32x4*>(p + k);
    return v;
  };
  for (int g0 = wave; g0 < groups; g0 += kFewWaves * kFewAhead) {
    i32x8 fb[kFewAhead], fa[kFewAhead][NT];
    float s[kFewAhead][NT];
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int g = g0 + u * kFewWaves;
      if (g < groups) fb[u] = both(chunk(b, g * kGroup), chunk(b, g * kGroup + 64));
    }
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int g = g0 + u * kFewWaves;
      if (g >= groups) continue;
      const float sb = b_scales[g];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        fa[u][t] = both(chunk(a[t], g * kGroup), chunk(a[t], g * kGroup + 64));
        s[u][t] = sb * c.a_scales[g * c.a_scale_stride + m_row[t]];
      }
    }
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      if (g0 + u * kFewWaves >= groups) continue;
      Operand<kWide> ob, oa;
      to_operand(fb[u], ob);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        to_operand(fa[u][t], oa);
        const floats4 p = group_product(ob, oa);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_fmaf(p[i], s[u][t], acc[t][i]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) parts[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < NT; t += kFewWaves) {
    floats4 sum = parts[0][t][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) sum += parts[w][t][lane];
    store_four(c, m0 + t * 16 + row, n0 + seg * 4, sum, BF16);
  }
}

// ---- many rows: tiles through LDS ------------------------------------------------------------------------------------------------
// A workgroup has BM rows of a and BN of b; a group of k of both is one stage in LDS (rows of 128 bytes, the 16-byte chunk c of
// row r at place c ^ (r & 7), so that 16 lanes reading one chunk of 16 rows meet all banks), with the rows' scales behind it.  STAGES of
// them in a ring: loads go straight to LDS, a stage is asked for STAGES - 1 turns before its use, and a wait is for the loads of
// one stage only.
template <int BM, int BN, int WM, int WN, int STAGES, int WAY, bool BF16>
__global__ __launch_bounds__(WM * WN * 64) void tiled_kernel(MatmulCall c, int tiles_m, int tiles_n) {
  constexpr int kWaves = WM * WN;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;          // tiles of a wavefront
  constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves;
  constexpr int kScaleBytes = kWaves * 256;
  constexpr int kStage = (BM + BN) * kGroup + kScaleBytes;
  static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && BN / WN <= kGroup && kWaves * 64 >= BM, "shape of a tile");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;

  // Workgroups go to the 8 XCDs in turn: each XCD gets a contiguous run of tiles, bands of 8 tiles of m one column of n after the other.
  const int total = tiles_m * tiles_n;
  int id = blockIdx.x;
  {
    const int per = total / 8, rest = total % 8, xcd = id & 7, at = id >> 3;
    id = xcd * per + (xcd < rest ? xcd : rest) + at;
  }
  constexpr int kBand = 8;
  const int band = id / (kBand * tiles_n), first_m = band * kBand;
  const int band_rows = tiles_m - first_m < kBand ? tiles_m - first_m : kBand;
  const int in_band = id - band * kBand * tiles_n;
  const int m0 = (first_m + in_band % band_rows) * BM, n0 = (in_band / band_rows) * BN;

  const int wm = wave / WN, wn = wave % WN;
  const int groups = (c.k + kGroup - 1) / kGroup;
  const char* a = static_cast<const char*>(c.a) + m0 * c.a_stride;
  const char* b = static_cast<const char*>(c.b) + n0 * c.b_stride;
  const int chunk = ((lane & 7) ^ (lane >> 3)) * 16;           // which bytes of its row's 128 a lane brings
  uint32_t row_at[kLoadsA + kLoadsB];
#pragma unroll
  for (int j = 0; j < kLoadsA + kLoadsB; ++j) {
    const bool is_a = j < kLoadsA;
    const int r = ((is_a ? j : j - kLoadsA) * kWaves + wave) * 8 + (lane >> 3);
    const int most = is_a ? c.m - 1 - m0 : c.n - 1 - n0;       // (rows past the end repeat the last one and are not stored)
    row_at[j] = (uint32_t)(r < most ? r : most) * (uint32_t)(is_a ? c.a_stride : c.b_stride);
  }
  const int scale_row = wave * 64 + lane;
  const float* a_scales = c.a_scales + m0;
  const int scale_at = scale_row < c.m - 1 - m0 ? scale_row : c.m - 1 - m0;

  auto issue = [&](int stage, int g) {
    const int k0 = g * kGroup;
    const uint32_t k = k0 + chunk < c.k ? k0 + chunk : 0;      // (bytes past the end of k are cleared in registers)
    char* to = lds + stage * kStage + wave * 1024;
#pragma unroll
    for (int j = 0; j < kLoadsA + kLoadsB; ++j) {
      const char* from = (j < kLoadsA ? a : b) + (row_at[j] + k);
      __builtin_amdgcn_global_load_lds((RLKV_GLOBAL void*)from, (RLKV_LDS void*)(to + j * kWaves * 1024), 16, 0, 0);
    }
    __builtin_amdgcn_global_load_lds((RLKV_GLOBAL void*)(a_scales + g * c.a_scale_stride + scale_at),
                                     (RLKV_LDS void*)(lds + stage * kStage + (BM + BN) * kGroup + wave * 256), 4, 0, 0);
  };
  constexpr int kLoads = kLoadsA + kLoadsB + 1;

  const float* b_scales = c.b_scales + ((n0 + wn * TN * 16) / kGroup < (c.n + kGroup - 1) / kGroup
                                            ? (n0 + wn * TN * 16) / kGroup : 0) * c.b_scale_stride;
  float sb_lanes = 0.f;                                        // the scales of 64 groups, one a lane

  const int row = lane & 15, seg = lane >> 4;
  const int at = row * kGroup + ((seg ^ (lane & 7)) << 4);
  const int at_a = (wm * TM * 16) * kGroup + at, at_b = (BM + wn * TN * 16) * kGroup + at;
  floats4 acc[TM][TN] = {};

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue(s, s < groups ? s : groups - 1);
  int stage = 0;
  auto turn = [&](int g, auto tail) {
    if ((g & 63) == 0) {
      sb_lanes = b_scales[g + lane < groups ? g + lane : groups - 1];
      asm volatile("" : "+v"(sb_lanes));                       // (waited for here, and not in every turn behind the loads to LDS)
    }
    // This stage's loads are in, of all wavefronts, and nobody reads the stage that is written next.
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads * (STAGES - 2)) : "memory");
    {
      const int next = g + STAGES - 1;                         // (past the end the last group once more: the count of loads stays)
      issue(stage == 0 ? STAGES - 1 : stage - 1, next < groups ? next : groups - 1);
    }
    const char* in = lds + stage * kStage;
    const float sb = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sb_lanes), g & 63));
    auto fragment = [&](int at_row) {
      i32x4 lo = *reinterpret_cast<const i32x4*>(in + at_row), hi = *reinterpret_cast<const i32x4*>(in + (at_row ^ 64));
      if constexpr (decltype(tail)::value) {                   // (chunks past the end of k)
        if (g * kGroup + seg * 16 >= c.k) lo = i32x4{0, 0, 0, 0};
        if (g * kGroup + seg * 16 + 64 >= c.k) hi = i32x4{0, 0, 0, 0};
      }
      Operand<WAY> o;
      to_operand(both(lo, hi), o);
      return o;
    };
    Operand<WAY> fb[TN], fa[2];
    floats4 p[2][TN];
    float s[TM];
    fa[0] = fragment(at_a);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = fragment(at_b + j * 16 * kGroup);
#pragma unroll
    for (int i = 0; i < TM; ++i)
      s[i] = *reinterpret_cast<const float*>(in + (BM + BN) * kGroup + (wm * TM * 16 + i * 16 + row) * 4);
#pragma unroll
    for (int i = 0; i <= TM; ++i) {
      // products of one tile row beside the sums of the row before: the matrix cores and the vector ALU both have work
      if (i + 1 < TM) fa[(i + 1) & 1] = fragment(at_a + (i + 1) * 16 * kGroup);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        if (i < TM) p[i & 1][j] = group_product(fb[j], fa[i & 1]);
        if (i > 0) {
          const float by = sb * s[i - 1];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i - 1][j][e] = __builtin_fmaf(p[(i - 1) & 1][j][e], by, acc[i - 1][j][e]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    stage = stage == STAGES - 1 ? 0 : stage + 1;
  };
  const int whole_groups = c.k / kGroup;
  for (int g = 0; g < whole_groups; ++g) turn(g, std::false_type{});
  if (whole_groups < groups) turn(whole_groups, std::true_type{});
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // (no load to LDS outlives the workgroup)
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
      store_four(c, m0 + (wm * TM + i) * 16 + row, n0 + (wn * TN + j) * 16 + seg * 4, acc[i][j], BF16);
}

template <int NT, bool BF16>
hipError_t launch_few(const MatmulCall& c, hipStream_t stream) {
  hipLaunchKernelGGL((few_rows_kernel<NT, BF16>), dim3((c.n + 15) / 16, (c.m + NT * 16 - 1) / (NT * 16)), dim3(kFewWaves * 64), 0, stream, c);
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int STAGES, int WAY, bool BF16>
hipError_t launch_tiled(const MatmulCall& c, hipStream_t stream) {
  const int tiles_m = (c.m + BM - 1) / BM, tiles_n = (c.n + BN - 1) / BN;
  constexpr int kLds = STAGES * ((BM + BN) * kGroup + WM * WN * 256);
  auto kernel = tiled_kernel<BM, BN, WM, WN, STAGES, WAY, BF16>;
  static const hipError_t allowed = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  if (allowed != hipSuccess) return allowed;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_m * tiles_n)), dim3(WM * WN * 64), kLds, stream, c, tiles_m, tiles_n);
  return hipGetLastError();
}

template <bool BF16>
hipError_t launch_typed(const MatmulCall& c, hipStream_t stream) {
  if (c.m <= 16) return launch_few<1, BF16>(c, stream);
  if (c.m <= 32) return launch_few<2, BF16>(c, stream);
  if (c.m <= 64) return launch_few<4, BF16>(c, stream);
  if constexpr (!BF16) return launch_tiled<128, 128, 2, 2, 4, kWide, false>(c, stream);
  const int64_t big = (int64_t)((c.m + 255) / 256) * ((c.n + 255) / 256);
  if (big >= 256) return launch_tiled<256, 256, 2, 4, 2, kFast, true>(c, stream);
  return launch_tiled<128, 128, 2, 2, 4, kFast, true>(c, stream);
}

}  // namespace

hipError_t launch_matmul(const MatmulCall& c, bool out_bf16, hipStream_t stream) {
  return out_bf16 ? launch_typed<true>(c, stream) : launch_typed<false>(c, stream);
}

}  // namespace rlkv
