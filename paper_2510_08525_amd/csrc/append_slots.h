// Which slots of a store an append touches and which of the new positions each of them gets; shared by the kernels that append.
#pragma once

#include "rlkv_internal.h"

namespace rlkv {

struct TileRange { int first, count; };

__device__ inline TileRange tiles_of(int slot_lo, int slot_hi /* exclusive */) {
  if (slot_hi <= slot_lo) return {0, 0};
  const int t0 = slot_lo / kTile, t1 = (slot_hi - 1) / kTile;
  return {t0, t1 - t0 + 1};
}

// Appended position that ends in `slot` after the append, or -1 if the slot is untouched.
__device__ inline int source_position(bool full, int slot, int len_old, int len_new, int S, int R) {
  int p;
  if (full || slot < S) {
    p = slot;
  } else {
    const int r = slot - S;
    if (r >= R) return -1;                       // padding slot behind the ring
    const int last = len_new - 1 - S;            // ring index space of the newest position
    if (last < r) return -1;
    p = S + r + R * ((last - r) / R);            // largest p < len_new with (p - S) % R == r
  }
  return (p >= len_old && p < len_new) ? p : -1;
}

// The tile of the store that the job-th workgroup of a pair works on, or -1 if the append touches fewer tiles.
__device__ inline int tile_of_job(bool full, int job, int len_old, int len_new, int S, int R) {
  if (full) {
    const TileRange t = tiles_of(len_old, len_new);
    return job < t.count ? t.first + job : -1;
  }
  // up to three slot ranges change: new sinks, and the ring range (which may wrap)
  const TileRange ta = tiles_of(len_old < S ? len_old : S, len_new < S ? len_new : S);
  const int p0 = len_old > S ? len_old : S;
  const int c = len_new - p0;                 // positions that go to the ring
  TileRange tb = {0, 0}, tc = {0, 0};
  if (c >= R) {
    tb = tiles_of(S, S + R);
  } else if (c > 0) {
    const int r0 = (p0 - S) % R;
    const int r1 = r0 + c;
    tb = tiles_of(S + r0, S + (r1 < R ? r1 : R));
    if (r1 > R) tc = tiles_of(S, S + r1 - R);
  }
  int j = job;
  if (j < ta.count) return ta.first + j;
  if ((j -= ta.count) < tb.count) return tb.first + j;
  if ((j -= tb.count) < tc.count) return tc.first + j;
  return -1;
}

// Workgroups of a pair that cover every tile an append of at most max_tokens tokens can touch: a range of c >= 1 slots touches at
// most (c + 30) / 32 + 1 tiles; a full head has one range, a compressed head up to three (new sinks, ring, wrapped
// ring) whose sizes add up to at most max_tokens.  One token touches one tile.
inline int append_jobs(int max_tokens) { return max_tokens <= 1 ? 1 : (max_tokens + 3 * (kTile - 2)) / kTile + 3; }

}  // namespace rlkv
