// Rotation of queries and keys by their positions: what the host hands to the kernels of rotary.hip.
#pragma once

#include <math.h>

#include "rlkv_internal.h"

namespace rlkv {

// Pair i of rotated columns turns by turn[i] / 2^64 of a full turn a position: position * turn, modulo 2^64, is the exact
// fraction of a turn at any position, with no argument too large to reduce.
struct RotaryTurns {
  uint64_t turn[kHeadDim / 2];
  int32_t pairs;                 // rotated columns / 2: a multiple of 8 (the columns past 2 * pairs stay as they are)
  int32_t interleaved;           // 1: pair i is columns 2 i and 2 i + 1; 0: columns i and i + pairs
};
// Those of a caller's frequencies; false where they are none.
inline bool turns_of(const rlkv_rotary_t* rotary, RotaryTurns* turns) {
  if (!rotary || !rotary->inv_freq) return false;
  const int pairs = rotary->n_pairs;
  if (pairs < 8 || pairs > kHeadDim / 2 || pairs % 8 != 0) return false;
  if (rotary->interleaved < 0 || rotary->interleaved > 1) return false;
  *turns = {};
  for (int i = 0; i < pairs; ++i) {
    if (!isfinite(rotary->inv_freq[i])) return false;
    // (whole turns do not matter, and what is left is below 1 unless it was rounded up to it)
    double t = rotary->inv_freq[i] * 0.15915494309189533577;          // 1 / (2 pi)
    t -= floor(t);
    turns->turn[i] = t < 1.0 ? (uint64_t)(t * 18446744073709551616.0) : 0;         // 2^64
  }
  turns->pairs = pairs;
  turns->interleaved = rotary->interleaved;
  return true;
}
struct RotaryCall {
  const void* qkv;               // [batch][stride_tokens] rows of token_stride elements: q heads, k heads, v heads of kHeadDim
  int64_t token_stride;
  int32_t stride_tokens;
  int32_t uniform;               // tokens of every active sequence, where no counts are given
  int32_t max_tokens;            // the largest count
  void* q_out;                   // [batch][n_q_heads][stride_tokens][kHeadDim], or null with an append: q is not wanted
  void* k_out;                   // [batch][n_kv_heads][stride_tokens][kHeadDim] (no append)
  void* v_out;
};
// `append`: the rotated keys and the values go into the layer's stores, lengths and list growth advance (as launch_append); else all
// three go out, heads first, and len_in and len_out are the two copies of the lengths, of which the larger is the present one (appends write
// theirs over the older copy, a step and a reset both): a recorded call finds it at every replay.  `seqs` non-null: per-sequence counts.
hipError_t launch_rotary(const DeviceView& dv, int layer, const int32_t* len_in, int32_t* len_out, const RotaryCall& call,
                         const RotaryTurns& turns, const SeqCounts* seqs, bool append, hipStream_t stream);

}  // namespace rlkv
