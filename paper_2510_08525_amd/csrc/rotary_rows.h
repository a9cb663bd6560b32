// Rotation of rows by their positions on the device.
//
// A pair (a, b) of columns at position p turns by the angle p * f:  (a cos - b sin, b cos + a sin).  The angle is a fraction of a turn in
// 32 bits of p * turn (rotary.h), exact at any position; its quadrant is two of those bits, and the rest, at most an eighth of a turn
// either way, goes through the Taylor series of sine and cosine (to x^9 and x^10: 2e-9 and 2e-10 there): 2e-7 of error in
// all with the roundings of fp32, and no table of positions to read.
//
// Eight threads hold a row: thread j two pieces of eight columns, those that turn together (j and j + pairs / 8, or 2 j and
// 2 j + 1), so all eight angles are its own.
#pragma once

#include "rotary.h"

namespace rlkv {

constexpr int kRowThreads = 8;

__device__ __forceinline__ void sin_cos_of_turn(uint32_t phase, float& sine, float& cosine) {
  const uint32_t quadrant = (phase + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(phase - (quadrant << 30)) * 1.46291807926715968e-9f;      // 2 pi / 2^32
  const float x2 = x * x;
  // (fused multiply-adds by name, here and in rotate: what the compiler fuses by itself differs between the kernels, and with it bits)
  float s = __builtin_fmaf(x2, 1.f / 362880, -1.f / 5040), c = __builtin_fmaf(x2, -1.f / 3628800, 1.f / 40320);
  s = __builtin_fmaf(x2, s, 1.f / 120);
  c = __builtin_fmaf(x2, c, -1.f / 720);
  s = __builtin_fmaf(x2, s, -1.f / 6);
  c = __builtin_fmaf(x2, c, 1.f / 24);
  c = __builtin_fmaf(x2, c, -0.5f);
  s = __builtin_fmaf(x * x2, s, x);
  c = __builtin_fmaf(x2, c, 1.f);
  const uint32_t flip_s = (quadrant & 2) << 30, flip_c = ((quadrant + 1) & 2) << 30;
  sine = __uint_as_float(__float_as_uint(quadrant & 1 ? c : s) ^ flip_s);
  cosine = __uint_as_float(__float_as_uint(quadrant & 1 ? s : c) ^ flip_c);
}

struct Angles { float sine[8], cosine[8]; };

__device__ __forceinline__ void turn_pair(float& x, float& y, float sine, float cosine) {
  const float a = x, b = y;
  x = __builtin_fmaf(a, cosine, -(b * sine));
  y = __builtin_fmaf(b, cosine, a * sine);
}

__device__ __forceinline__ void angles_of(const RotaryTurns& turns, int j, uint32_t position, Angles& a) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t turn = turns.turn[j * 8 + i];
    const uint32_t phase = position * (uint32_t)(turn >> 32) + __umulhi(position, (uint32_t)turn);
    sin_cos_of_turn(phase, a.sine[i], a.cosine[i]);
  }
}

// The two pieces of thread j of a row, and their rotation (j < pairs / 8; the others stay as they are).
__device__ __forceinline__ int first_piece(const RotaryTurns& t, int j) { return !t.interleaved && j < t.pairs / 8 ? j : 2 * j; }
__device__ __forceinline__ int second_piece(const RotaryTurns& t, int j) {
  return !t.interleaved && j < t.pairs / 8 ? j + t.pairs / 8 : 2 * j + 1;
}
__device__ __forceinline__ void rotate(const RotaryTurns& t, const Angles& g, float (&a)[8], float (&b)[8]) {
  if (!t.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair(a[i], b[i], g.sine[i], g.cosine[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn_pair(a[2 * i], a[2 * i + 1], g.sine[i], g.cosine[i]);
      turn_pair(b[2 * i], b[2 * i + 1], g.sine[4 + i], g.cosine[4 + i]);
    }
  }
}

}  // namespace rlkv
