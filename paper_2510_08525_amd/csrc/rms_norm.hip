// Root-mean-square norm of rows with the addition of a residual, into the storage type or into 8 bits with a scale for each group
// of 128 columns; quantising alone is the same kernel without the norm.
//
//   h = x + r          y = h / sqrt(mean(h^2) + eps) * w          s_g = max(max_g |y| / 448, least)      out = round(y / s_g)
//
// h stays in fp32 registers between the sum of squares and the outputs, so it is read once and each output is rounded once: the norm is
// that of the unrounded sum.  A thread has one piece of eight columns (two beyond 8192 columns, and what is beyond 16384 is read a
// second time): all of a row's pieces are asked for at once, a wavefront's are whole lines, and the 16 lanes of a group of 128 columns
// lie next to each other, so that its maximum takes four steps over lanes and no LDS.
// Bound: HBM for many rows (16384 x 3584 bf16 with residual into 8 bits: 413 MB in 75 to 77 us, 5.4 to 5.5 TB/s; a copy of 1 GiB reaches 5.05), latency for few
// (one row of 4096: 4 us, the kernel 2.9): x, in bf16 the residual behind it (each is widened as it arrives), and the weight behind the sum.
// With 64 threads a row and eight pieces each, weights kept over several rows, the same call took 134 us, with 256 threads and two pieces 90
// (both with plain accesses); several rows to a workgroup one after the other are slower in every shape.
#include <type_traits>

#include "token_ops.h"

namespace rlkv {
namespace {

// T threads a row, NC pieces each (T * NC * 8 columns at most, unless LOOP: then the pieces beyond are read a second time).
template <typename X, int T, int NC, bool E4M3, bool LOOP, bool STREAM>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_kernel(NormCall c) {
  constexpr int kRowsAtOnce = T < 256 ? 256 / T : 1;
  constexpr int kWaves = T / 64;
  __shared__ float parts[2][kWaves > 1 ? kWaves : 1];
  const int t = threadIdx.x % T, lane_row = threadIdx.x / T;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRowsAtOnce + lane_row; row < c.rows; row += (int64_t)gridDim.x * kRowsAtOnce) {
    const X* x = static_cast<const X*>(c.x) + row * c.x_stride;
    const X* res = c.residual ? static_cast<const X*>(c.residual) + row * c.residual_stride : nullptr;
    float h[NC][8];
    float squares = 0.f;
    auto load = [&](int col, float (&f)[8]) {
      load_piece<STREAM>(x, col, c.cols, f);
      if (res) {
        float r[8];
        load_piece<STREAM>(res, col, c.cols, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += r[i];
      }
    };
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int col = (t + k * T) * 8;
      if (col < c.cols) {
        load(col, h[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k][i] = 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += h[k][i] * h[k][i];
    float factor = 1.f;
    if (c.norm) {
      if (LOOP)
        for (int col = (t + NC * T) * 8; col < c.cols; col += T * 8) {
          float f[8];
          load(col, f);
#pragma unroll
          for (int i = 0; i < 8; ++i) squares += f[i] * f[i];
        }
      squares = sum_of_wave(squares);
      if (kWaves > 1) {
        // (two buffers in turn: a wavefront may be at the next row while another still reads this one's sums)
        if ((threadIdx.x & 63) == 0) parts[turn][threadIdx.x >> 6] = squares;
        __syncthreads();
        squares = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) squares += parts[turn][w];
        turn ^= 1;
      }
      factor = rsqrtf(squares / (float)c.cols + c.eps);
    }
    auto finish = [&](int col, float (&f)[8]) {
      if (col < c.cols) {
        if (c.sum_out) store_piece<STREAM>(static_cast<X*>(c.sum_out) + row * c.sum_stride, col, c.cols, f);
        if (c.norm) {
          float w[8];
          if (c.weight) {
            load_piece(static_cast<const X*>(c.weight), col, c.cols, w);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 1.f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = f[i] * factor * w[i];
        }
      }
      if constexpr (E4M3) {
        // the lanes of a group are 16 neighbours, those past the row's end among them (with zeros)
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(f[i]));
        most = fmaxf(most, from_lane<0x128, 0xf>(0.f, most));          // row_ror:8, 4, 2, 1
        most = fmaxf(most, from_lane<0x124, 0xf>(0.f, most));
        most = fmaxf(most, from_lane<0x122, 0xf>(0.f, most));
        most = fmaxf(most, from_lane<0x121, 0xf>(0.f, most));
        const float scale = fmaxf(most / kE4m3Max, kLeastScale);
        if (col < c.cols) {
          // The quotient, as a product with the reciprocal in two parts (the second is what the first leaves of 1 / scale, and not negative, so
          // that -0 stays -0): rounded once, where the rounded reciprocal alone puts two roundings next to a tie.
          float inverse = 1.f / scale, left = __builtin_fmaf(-inverse, scale, 1.f);
          if (left < 0.f) {
            inverse = __uint_as_float(__float_as_uint(inverse) - 1);
            left = __builtin_fmaf(-inverse, scale, 1.f);
          }
          const float rest = scale < INFINITY ? left * inverse : 0.f;          // (an infinite scale: 0, and NaN of an infinity)
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = __builtin_fmaf(f[i], inverse, f[i] * rest);
          store_e4m3(static_cast<uint8_t*>(c.out) + row * c.out_stride, col, c.cols, f);
          if ((t & 15) == 0) c.scales[(int64_t)(col / kGroup) * c.scale_stride + row] = scale;
        }
      } else if (col < c.cols) {
        store_piece<STREAM>(static_cast<X*>(c.out) + row * c.out_stride, col, c.cols, f);
      }
    };
    if (LOOP)                       // (before the pieces in registers: where sum_out is the residual, what is read again here is not yet written)
      for (int col = (t + NC * T) * 8; col - t * 8 < c.cols; col += T * 8) {
        float f[8] = {};
        if (col < c.cols) load(col, f);
        finish(col, f);
      }
#pragma unroll
    for (int k = 0; k < NC; ++k) finish((t + k * T) * 8, h[k]);
  }
}

constexpr int kMostBlocks = 1 << 20;

// (STREAM: 8-bit outputs, which the product behind the norm reads, are not meant.)
template <typename X, bool E4M3, bool STREAM>
hipError_t launch_typed(const NormCall& c, hipStream_t stream) {
  auto run = [&](auto kernel, int threads, int rows_at_once) {
    const int blocks = (int)(((int64_t)c.rows + rows_at_once - 1) / rows_at_once);
    hipLaunchKernelGGL(kernel, dim3(blocks < kMostBlocks ? blocks : kMostBlocks), dim3(threads), 0, stream, c);
    return hipGetLastError();
  };
  if (c.cols <= 512) return run(norm_kernel<X, 64, 1, E4M3, false, STREAM>, 256, 4);
  if (c.cols <= 2048) return run(norm_kernel<X, 256, 1, E4M3, false, STREAM>, 256, 1);
  if (c.cols <= 4096) return run(norm_kernel<X, 512, 1, E4M3, false, STREAM>, 512, 1);
  if (c.cols <= 8192) return run(norm_kernel<X, 1024, 1, E4M3, false, STREAM>, 1024, 1);
  return run(norm_kernel<X, 1024, 2, E4M3, true, STREAM>, 1024, 1);
}

}  // namespace

hipError_t launch_norm(const NormCall& c, int dtype, bool out_e4m3, hipStream_t stream) {
  // (us, plain accesses / non-temporal ones, bf16 with residual into 8 bits: 16384 x 3584 80.4 / 76.4; 8192 x 3584, which a
  // cache holds, 43.2 / 39.9 by itself: not taken)
  const int64_t bytes = dtype == RLKV_F32 ? 4 : 2;
  const bool through = c.rows * (int64_t)c.cols * (bytes * (1 + (c.residual != nullptr) + (c.sum_out != nullptr)) + (out_e4m3 ? 1 : bytes)) > kStreamBytes;
  auto launch = [&](auto x, auto e4m3) {
    typedef decltype(x) X;
    constexpr bool E4M3 = decltype(e4m3)::value;
    return through ? launch_typed<X, E4M3, true>(c, stream) : launch_typed<X, E4M3, false>(c, stream);
  };
  if (dtype == RLKV_F32) return out_e4m3 ? launch(float(), std::true_type{}) : launch(float(), std::false_type{});
  return out_e4m3 ? launch(uint16_t(), std::true_type{}) : launch(uint16_t(), std::false_type{});
}

}  // namespace rlkv
