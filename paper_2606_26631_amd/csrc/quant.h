// The decoder cache in 8 bits: parameter blocks, launchers, and the device side of its codes.
//
// A row (one slot, layer and KV head) is head_dim codes and a float32 scale.  With x the row
// that a cache of the inputs' type would hold and Q the largest code, in float32:
//   scale = max(max |x_i| / Q, 2^-126),   code_i = nearest(x_i (1 / scale)), ties to even
// and the row stands for code_i scale.  A row with an infinity or a NaN has codes 0 and scale NaN.
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

#include "prcr_internal.h"

namespace prcr {

// Where a cache's rows are.  Of the slot `base` stands for (place_of), layer l's and head h's row
// is base + l layer_rows + h head_rows, its scale the same with layer_scales and head_scales.
struct QuantStore {
  void *k, *v;                    // codes
  float *k_scale, *v_scale;
  const int32_t *block_table;
  int64_t layer_rows, layer_scales;
  int32_t head_rows, head_scales;
  int32_t paged, code;
  int32_t n_layers, n_kv_heads, s_max, block_size, max_blocks, n_blocks;
  Divisor by_block;
};

struct QuantWriteParams {
  QuantStore to;
  const void *k, *v;              // [batch][s_src][n_kv_heads][head_dim], or a memory's rows
  const int32_t *pos;             // append: [batch][s_src][3]
  const int32_t *n_tokens;        // append: [batch]
  const int32_t *start;           // [batch]: cache_start or cache_len
  const int32_t *sel_off, *sel_idx, *n_visual, *v_slot;   // rebind (v_slot: of a memory without values)
  const double *new_pos;
  int32_t *new_len;
  int64_t *slot_mapping;
  int32_t *err;
  int32_t batch, s_src, max_visual, layer;
  int32_t n_tok;                  // tokens: batch * s_src, or total_k
  int32_t rows;                   // (layer, head) rows of a token: n_kv_heads, or n_layers * n_kv_heads
  int32_t rows_per_group;         // of those, a workgroup's (launcher)
  Divisor by_seq, by_heads;
  uint64_t on_h, on_w;            // pairs that turn by the h and by the w position (the others: t)
  double inv_freq[kMaxPairs];
};

struct QuantReadParams {
  QuantStore from;
  void *k, *v;                    // out [batch][1][n_kv_heads][s_out][head_dim]
  const int32_t *cache_len;
  int32_t *err;
  int32_t batch, layer, s_out, capacity;
  Divisor by_heads, by_chunk;     // (launcher)
};

struct QuantDecodeParams : DecodeParams {
  const float *k_scale, *v_scale;
  int32_t q_f32;                  // the queries' type
  int32_t heads;                  // KV heads of a workgroup (launcher)
};

hipError_t launch_quant_append(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream);
hipError_t launch_quant_rebind(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream);
hipError_t launch_quant_read(const QuantReadParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream);
hipError_t launch_quant_decode(const QuantDecodeParams &p, prcr_code code, int head_dim, bool paged, hipStream_t stream);

#ifdef __HIPCC__
namespace {

// Where a sequence's slot lies: in two steps, so that a paged cache's table entry, read from a
// clamped place (always in the table), can be on its way with other loads.
struct SlotEntry {
  int64_t slot;
  int64_t lb;                     // paged: the logical block, -1 outside the table
  int32_t blk;                    // and its entry
};
__device__ __forceinline__ SlotEntry entry_of_slot(const QuantStore &s, int b, int64_t slot) {
  SlotEntry e{slot, 0, 0};
  if (s.paged) {
    const bool in = slot >= 0 && slot < static_cast<int64_t>(s.max_blocks) * s.block_size;   // (at most 2^30)
    e.lb = in ? static_cast<int64_t>(s.by_block.divide(static_cast<uint32_t>(slot))) : -1;
    e.blk = s.block_table[static_cast<int64_t>(b) * s.max_blocks + (in ? e.lb : 0)];
  }
  return e;
}
// Bases of the slot; flag: what is wrong with it (then they are not to be used).
struct Place {
  int64_t row, scale;
  int64_t id;                     // contiguous b s_max + slot, paged block block_size + offset
  int flag;
};
__device__ __forceinline__ Place place_of(const QuantStore &s, int b, const SlotEntry &e) {
  Place at{0, 0, -1, 0};
  if (s.paged) {
    const int64_t off = e.slot - e.lb * s.block_size;
    at.flag = e.lb < 0 ? PRCR_DERR_CAPACITY : (e.blk >= 0 && e.blk < s.n_blocks ? 0 : PRCR_DERR_BLOCK);
    at.id = static_cast<int64_t>(e.blk) * s.block_size + off;
    at.row = at.id * s.n_kv_heads;
    at.scale = static_cast<int64_t>(e.blk) * s.n_kv_heads * s.block_size + off;
  } else {
    at.flag = e.slot >= 0 && e.slot < s.s_max ? 0 : PRCR_DERR_CAPACITY;
    at.id = static_cast<int64_t>(b) * s.s_max + e.slot;
    at.row = at.scale = static_cast<int64_t>(b) * s.n_layers * s.n_kv_heads * s.s_max + e.slot;
  }
  return at;
}

// The numbers that a word's four codes stand for, before the scale.
__device__ __forceinline__ void decode4(uint32_t w, bool e4m3, float *x) {
  if (e4m3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = static_cast<float>(static_cast<int8_t>(w >> (8 * e)));
  }
}

}  // namespace
#endif

}  // namespace prcr
