// Packed projections of a token -> rotated queries and keys, and on the way the append of keys and values to the head-mixed cache.
//
// The rotation is that of rotary_rows.h.  Queries: a thread keeps its token's sines and cosines over several heads.  Keys and
// values of an append: one workgroup per tile of 32 slots (destination driven, like append_kernel), whose row pieces pass through LDS into
// the tile.  Bound: HBM for prompts (8 x 2000 tokens of 32 / 8 heads handed out heads first: 393 MB in 70.6 us, 5.6 TB/s), one chain of memory
// latencies for a single token.
#include <type_traits>

#include "append_slots.h"
#include "rotary.h"
#include "rotary_rows.h"
#include "tile_rows.h"
#include "token_ops.h"

namespace rlkv {
namespace {

constexpr int kItems = kBlock / kRowThreads;       // rows a workgroup works on side by side: those of a tile

template <int KERNEL, typename T, bool APPEND, bool STREAM>
__global__ __launch_bounds__(kBlock) void rotary_kernel(DeviceView dv, int layer, const int32_t* __restrict__ len_in,
                                                        int32_t* __restrict__ len_out, RotaryCall call, RotaryTurns turns, int ragged,
                                                        SeqCounts seqs, int jobs, int heads_each) {
  const T* qkv = static_cast<const T*>(call.qkv);
  const int Hq = dv.n_q_heads, H = dv.n_kv_heads;
  const int item = threadIdx.x / kRowThreads, j = threadIdx.x % kRowThreads;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const bool turned = j < turns.pairs / 8;
  const int n_append = APPEND ? dv.n_pairs * jobs : 0;
  auto tokens_of = [&](int b) { return ragged ? tokens_of_seq(dv, seqs, b) : (dv.active[b] ? call.uniform : 0); };

  if (APPEND && (int)blockIdx.x < n_append) {
    const int pair = blockIdx.x / jobs, job = blockIdx.x % jobs, b = pair / H, h = pair % H;
    const int S = dv.sink, R = dv.recent;
    const int n_tok = tokens_of(b);
    const int len_old = len_in[b], len_new = len_old + n_tok;
    if (job == 0 && h == 0 && threadIdx.x == 0) len_out[b] = len_new;
    if (!ragged && blockIdx.x == 0 && threadIdx.x == 0) list_header(dv, layer)->grow += call.uniform;
    const bool full = dv.full_mask[layer * H + h] != 0;
    const int tile = n_tok > 0 ? tile_of_job(full, job, len_old, len_new, S, R) : -1;
    if (tile < 0) return;
    const int64_t koff = dv.store_off[((int64_t)layer * dv.batch + b) * H + h];
    const int slot = tile * kTile + item;
    const int p = source_position(full, slot, len_old, len_new, S, R);
    if (!full && j == 0 && p >= 0) dv.slot_pos[dv.slotpos_off[layer * H + h] + (int64_t)b * dv.window + slot] = p;
    float k0[8], k1[8], v0[8], v1[8];
    if (p >= 0) {
      const T* row = qkv + ((int64_t)b * call.stride_tokens + (p - len_old)) * call.token_stride + (int64_t)(Hq + h) * kHeadDim;
      load_piece<STREAM>(row, c0, kHeadDim, k0);
      load_piece<STREAM>(row, c1, kHeadDim, k1);
      load_piece<STREAM>(row + (int64_t)H * kHeadDim, c0, kHeadDim, v0);
      load_piece<STREAM>(row + (int64_t)H * kHeadDim, c1, kHeadDim, v1);
      if (turned) {
        Angles g;
        angles_of(turns, j, (uint32_t)p, g);
        rotate(turns, g, k0, k1);
      }
    }
    if constexpr (KERNEL == RLKV_KERNEL_MFMA) {
      __shared__ TileRowsLds lds;
      __shared__ int32_t have[kTile];
      if (j == 0) have[item] = p >= 0;
      bool wide = false;
      if (p >= 0) {
        Piece<uint16_t> piece;
        auto put_k = [&](const float (&f)[8], int col) {
          narrow(f, piece);
          lds.k[k_unit(item, col >> 3)] = __builtin_bit_cast(uint4, piece.w);
        };
        auto put_v = [&](const float (&f)[8], int col) {
          narrow(f, piece);
          *reinterpret_cast<words4*>(lds.v + item * kTileRowStride + col * 2) = piece.w;
#pragma unroll
          for (int i = 0; i < 4; ++i) wide |= any_beyond_fp16(piece.w[i]);
        };
        put_k(k0, c0); put_k(k1, c1);
        put_v(v0, c0); put_v(v1, c1);
      }
      __syncthreads();
      char* base = dv.kv_base + koff + (int64_t)tile * kTileBytes;
      if (full && dv.page_shift >= 0)
        base = dv.kv_base + koff + dv.block_table[(int64_t)b * dv.table_stride + (tile >> dv.page_shift)] * dv.page_bytes +
               (int64_t)(tile & dv.page_mask) * kTileBytes;
      tile_from_lds<true>(lds, [&](int s) { return have[s] == 0; }, base);
      if (wide) dv.v_wide[layer] = 1;        // the prefill kernel takes this layer's V as bf16 from now on
    } else if (p >= 0) {
      const int cap = full ? dv.cap_pad[b] : dv.window_pad;
      T* krow = reinterpret_cast<T*>(dv.kv_base + koff + (int64_t)slot * dv.row_bytes);
      T* vrow = reinterpret_cast<T*>(dv.kv_base + koff + (int64_t)(cap + slot) * dv.row_bytes);
      store_piece(krow, c0, kHeadDim, k0);
      store_piece(krow, c1, kHeadDim, k1);
      store_piece(vrow, c0, kHeadDim, v0);
      store_piece(vrow, c1, kHeadDim, v1);
    }
    return;
  }

  // Rows that go out: of the queries, and without an append of keys and values too.
  const int n_heads = APPEND ? Hq : Hq + 2 * H;
  const int parts = (n_heads + heads_each - 1) / heads_each;
  const int64_t index = (int64_t)(blockIdx.x - n_append) * kItems + item;
  const int64_t token = index / parts;
  if (token >= (int64_t)dv.batch * call.max_tokens) return;
  const int b = (int)(token / call.max_tokens), c = (int)(token % call.max_tokens);
  const int n_tok = ragged ? (seqs.in_args ? seqs.tok[b] : dv.append_cnt[b]) : (dv.active[b] ? call.uniform : 0);
  if (c >= n_tok) return;
  const int h_first = (int)(index % parts) * heads_each;
  const int h_last = h_first + heads_each < n_heads ? h_first + heads_each : n_heads;
  const T* row = qkv + ((int64_t)b * call.stride_tokens + c) * call.token_stride;
  Angles g = {};
  int n = len_in[b];
  if constexpr (!APPEND) {
    const int other = len_out[b];
    n = other > n ? other : n;
  }
  if (turned && h_first < Hq + H) angles_of(turns, j, (uint32_t)(n + c), g);
  for (int h = h_first; h < h_last; ++h) {
    float x[8], y[8];
    load_piece<STREAM>(row + (int64_t)h * kHeadDim, c0, kHeadDim, x);
    load_piece<STREAM>(row + (int64_t)h * kHeadDim, c1, kHeadDim, y);
    if (turned && h < Hq + H) rotate(turns, g, x, y);
    T* out = h < Hq ? static_cast<T*>(call.q_out) + ((int64_t)b * Hq + h) * call.stride_tokens * kHeadDim
             : h < Hq + H ? static_cast<T*>(call.k_out) + ((int64_t)b * H + h - Hq) * call.stride_tokens * kHeadDim
                          : static_cast<T*>(call.v_out) + ((int64_t)b * H + h - Hq - H) * call.stride_tokens * kHeadDim;
    out += (int64_t)c * kHeadDim;
    store_piece<STREAM>(out, c0, kHeadDim, x);
    store_piece<STREAM>(out, c1, kHeadDim, y);
  }
}

// One token a sequence (a decode step): the same work laid out for latency.  Eight threads have a query head's row, or a KV head's key and
// value row; the rows are asked for before anything that says where they go (fp32 rows are still under way then, bf16 ones, widened as they arrive,
// are waited for), and a row's pieces are stored from registers.
constexpr int kStepBlock = 64;
template <int KERNEL, typename T>
__global__ __launch_bounds__(kStepBlock) void rotary_step_kernel(DeviceView dv, int layer, const int32_t* __restrict__ len_in,
                                                                 int32_t* __restrict__ len_out, RotaryCall call, RotaryTurns turns, int ragged,
                                                                 SeqCounts seqs, int first_head) {
  const int Hq = dv.n_q_heads, H = dv.n_kv_heads, heads = Hq + H - first_head;
  const int index = blockIdx.x * (kStepBlock / kRowThreads) + threadIdx.x / kRowThreads, j = threadIdx.x % kRowThreads;
  const int b = index / heads, head = first_head + index % heads, h = head - Hq;
  if (b >= dv.batch) return;
  const int c0 = first_piece(turns, j) * 8, c1 = second_piece(turns, j) * 8;
  const T* row = static_cast<const T*>(call.qkv) + (int64_t)b * call.stride_tokens * call.token_stride + (int64_t)head * kHeadDim;
  float x[8], y[8], v0[8], v1[8];
  load_piece(row, c0, kHeadDim, x);
  load_piece(row, c1, kHeadDim, y);
  if (h >= 0) {
    load_piece(row + (int64_t)H * kHeadDim, c0, kHeadDim, v0);
    load_piece(row + (int64_t)H * kHeadDim, c1, kHeadDim, v1);
  }
  const int n = len_in[b];
  const bool there = ragged ? (seqs.in_args ? seqs.tok[b] : dv.append_cnt[b]) != 0 : dv.active[b] != 0;
  if (h == 0 && j == 0) len_out[b] = n + there;
  if (!ragged && b == 0 && h == 0 && j == 0) list_header(dv, layer)->grow += 1;
  if (!there) return;
  if (j < turns.pairs / 8) {
    Angles g;
    angles_of(turns, j, (uint32_t)n, g);
    rotate(turns, g, x, y);
  }
  if (h < 0) {
    T* out = static_cast<T*>(call.q_out) + ((int64_t)b * Hq + head) * call.stride_tokens * kHeadDim;
    store_piece(out, c0, kHeadDim, x);
    store_piece(out, c1, kHeadDim, y);
    return;
  }
  const bool full = dv.full_mask[layer * H + h] != 0;
  const int S = dv.sink, slot = full || n < S ? n : S + (n - S) % dv.recent;
  if (!full && j == 0) dv.slot_pos[dv.slotpos_off[layer * H + h] + (int64_t)b * dv.window + slot] = n;
  char* store = dv.kv_base + dv.store_off[((int64_t)layer * dv.batch + b) * H + h];
  if constexpr (KERNEL == RLKV_KERNEL_MFMA) {
    const int tile = slot / kTile, s = slot % kTile, s16 = s & 15;
    char* base = store + (int64_t)tile * kTileBytes;
    if (full && dv.page_shift >= 0)
      base = store + dv.block_table[(int64_t)b * dv.table_stride + (tile >> dv.page_shift)] * dv.page_bytes +
             (int64_t)(tile & dv.page_mask) * kTileBytes;
    // K: [half][chunk][slot % 16]; V: [d / 16][kb][d % 16][e] (rlkv_internal.h)
    const int kb = (s16 >> 2), e = (s >> 4) * 4 + (s & 3);
    bool wide = false;
    auto put = [&](const float (&k)[8], const float (&v)[8], int col) {
      Piece<uint16_t> piece;
      narrow(k, piece);
      *reinterpret_cast<words4*>(base + (s >> 4) * 4096 + (col >> 3) * 256 + s16 * 16) = piece.w;
      narrow(v, piece);
      uint16_t* to = reinterpret_cast<uint16_t*>(base + kTileBytes / 2) + (((col >> 4) * 4 + kb) * 16 + (col & 15)) * 8 + e;
#pragma unroll
      for (int i = 0; i < 8; ++i) to[i * 8] = (uint16_t)(piece.w[i >> 1] >> (16 * (i & 1)));
#pragma unroll
      for (int i = 0; i < 4; ++i) wide |= any_beyond_fp16(piece.w[i]);
    };
    put(x, v0, c0);
    put(y, v1, c1);
    if (wide) dv.v_wide[layer] = 1;        // the prefill kernel takes this layer's V as bf16 from now on
  } else {
    const int cap = full ? dv.cap_pad[b] : dv.window_pad;
    T* krow = reinterpret_cast<T*>(store + (int64_t)slot * dv.row_bytes);
    T* vrow = reinterpret_cast<T*>(store + (int64_t)(cap + slot) * dv.row_bytes);
    store_piece(krow, c0, kHeadDim, x);
    store_piece(krow, c1, kHeadDim, y);
    store_piece(vrow, c0, kHeadDim, v0);
    store_piece(vrow, c1, kHeadDim, v1);
  }
}

template <int KERNEL, typename T, bool APPEND>
hipError_t launch_typed(const DeviceView& dv, int layer, const int32_t* len_in, int32_t* len_out, const RotaryCall& call,
                        const RotaryTurns& turns, const SeqCounts* seqs, hipStream_t stream) {
  const SeqCounts none = {};
  if constexpr (APPEND) {
    if (call.max_tokens == 1) {
      const int first_head = call.q_out ? 0 : dv.n_q_heads;
      const int64_t threads = (int64_t)dv.batch * (dv.n_q_heads + dv.n_kv_heads - first_head) * kRowThreads;
      hipLaunchKernelGGL((rotary_step_kernel<KERNEL, T>), dim3((unsigned)((threads + kStepBlock - 1) / kStepBlock)), dim3(kStepBlock), 0, stream,
                         dv, layer, len_in, len_out, call, turns, seqs != nullptr, seqs ? *seqs : none, first_head);
      return hipGetLastError();
    }
  }
  const int n_heads = APPEND ? (call.q_out ? dv.n_q_heads : 0) : dv.n_q_heads + 2 * dv.n_kv_heads;
  const int jobs = append_jobs(call.max_tokens);
  const int64_t tokens = (int64_t)dv.batch * call.max_tokens;
  const int heads_each = tokens >= 1024 ? 8 : 1;
  const int64_t items = n_heads ? tokens * ((n_heads + heads_each - 1) / heads_each) : 0;
  const int64_t blocks = (APPEND ? (int64_t)dv.n_pairs * jobs : 0) + (items + kItems - 1) / kItems;
  if (blocks * kBlock > 0xffffffffll) return hipErrorInvalidValue;      // threads of a launch
  // (32 prompts of 200 .. 1500 tokens, 32 / 8 heads, with reset and a step: 162 us with plain accesses, 157.7 with non-temporal ones, 167.9 with
  // non-temporal loads alone)
  const int64_t values = tokens * (dv.n_q_heads + 2 * dv.n_kv_heads + n_heads) * kHeadDim;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, dv, layer, len_in, len_out, call, turns, seqs != nullptr,
                       seqs ? *seqs : none, jobs, heads_each);
    return hipGetLastError();
  };
  return values * (int64_t)sizeof(T) > kStreamBytes ? launch(rotary_kernel<KERNEL, T, APPEND, true>) : launch(rotary_kernel<KERNEL, T, APPEND, false>);
}

}  // namespace

hipError_t launch_rotary(const DeviceView& dv, int layer, const int32_t* len_in, int32_t* len_out, const RotaryCall& call,
                         const RotaryTurns& turns, const SeqCounts* seqs, bool append, hipStream_t stream) {
  if (dv.dtype == RLKV_F32)
    return append ? launch_typed<RLKV_KERNEL_VALU, float, true>(dv, layer, len_in, len_out, call, turns, seqs, stream)
                  : launch_typed<RLKV_KERNEL_VALU, float, false>(dv, layer, len_in, len_out, call, turns, seqs, stream);
  if (!append) return launch_typed<RLKV_KERNEL_VALU, uint16_t, false>(dv, layer, len_in, len_out, call, turns, seqs, stream);
  return dv.kernel == RLKV_KERNEL_MFMA
             ? launch_typed<RLKV_KERNEL_MFMA, uint16_t, true>(dv, layer, len_in, len_out, call, turns, seqs, stream)
             : launch_typed<RLKV_KERNEL_VALU, uint16_t, true>(dv, layer, len_in, len_out, call, turns, seqs, stream);
}

}  // namespace rlkv
