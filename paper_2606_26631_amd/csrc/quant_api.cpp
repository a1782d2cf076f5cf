// extern "C" entry points of the decoder cache in 8 bits: structural validation on the host,
// then the launches on the caller's stream.  No entry point allocates or keeps state.
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "quant.h"

using namespace prcr;

namespace {

constexpr int64_t kMaxSlots = int64_t{1} << 30;    // cache capacity per sequence

bool aligned(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct Range {
  const void *at;
  double bytes;
};
// Whether two byte ranges share a byte (null never does).
bool overlap(const Range &x, const Range &y) {
  if (x.at == nullptr || y.at == nullptr || !(x.bytes > 0) || !(y.bytes > 0)) return false;
  const double a = static_cast<double>(reinterpret_cast<uintptr_t>(x.at));
  const double b = static_cast<double>(reinterpret_cast<uintptr_t>(y.at));
  return a < b + y.bytes && b < a + x.bytes;
}
// Whether any of `written` shares memory with one of `read`, or with another of itself.
template <int kWritten, int kRead>
bool aliases(const Range (&written)[kWritten], const Range (&read)[kRead]) {
  for (int i = 0; i < kWritten; ++i) {
    for (const Range &r : read)
      if (overlap(written[i], r)) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return true;
  }
  return false;
}

int elem_bytes(prcr_dtype d) { return d == PRCR_F32 ? 4 : 2; }

prcr_status check_rope(const prcr_rope *rope, AxisMapId *map) {
  if (rope == nullptr) return PRCR_ERR_NULL;
  const int d = rope->head_dim;
  if (d < 2 || d % 2 != 0 || d / 2 > kMaxPairs) return PRCR_ERR_SHAPE;
  for (int a = 0; a < 3; ++a)
    if (rope->section[a] < 0) return PRCR_ERR_SHAPE;
  if (static_cast<int64_t>(rope->section[0]) + rope->section[1] + rope->section[2] != d / 2) return PRCR_ERR_SHAPE;
  if (rope->interleaved != 0 && rope->interleaved != 1) return PRCR_ERR_SHAPE;
  if (!(rope->theta > 0.0) || !std::isfinite(rope->theta)) return PRCR_ERR_SHAPE;
  *map = axis_map_id(*rope);
  return *map == AxisMapId::kUnsupported ? PRCR_ERR_UNSUPPORTED : PRCR_OK;
}

prcr_status check_dtype(prcr_dtype dtype) { return dtype == PRCR_F32 || dtype == PRCR_BF16 ? PRCR_OK : PRCR_ERR_DTYPE; }

// Code, layout flag and geometry of a cache; the slots a sequence has.
prcr_status cache_shape(const prcr_quant_cache *cache, int64_t *capacity) {
  if (cache == nullptr) return PRCR_ERR_NULL;
  if (cache->code != PRCR_E4M3 && cache->code != PRCR_I8) return PRCR_ERR_DTYPE;
  const prcr_cache &c = cache->cache;
  if (c.paged != 0 && c.paged != 1) return PRCR_ERR_SHAPE;
  if (c.paged) {
    if (c.block_size < 1 || c.max_blocks < 1 || c.n_blocks < 1) return PRCR_ERR_SHAPE;
    *capacity = static_cast<int64_t>(c.max_blocks) * c.block_size;
  } else {
    if (c.s_max < 1) return PRCR_ERR_SHAPE;
    *capacity = c.s_max;
  }
  return *capacity > kMaxSlots ? PRCR_ERR_SHAPE : PRCR_OK;
}

// The whole of a cache: its geometry, the shape it is used in, its pointers.
prcr_status check_cache(const prcr_quant_cache *cache, int32_t batch, int32_t n_layers, int32_t n_kv_heads,
                        int32_t head_dim, int64_t *capacity) {
  prcr_status st = cache_shape(cache, capacity);
  if (st != PRCR_OK) return st;
  if (batch < 1 || batch > 65535 || n_layers < 1 || n_kv_heads < 1 || n_kv_heads > 65535) return PRCR_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return PRCR_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(n_layers) * n_kv_heads > INT32_MAX / 2) return PRCR_ERR_SHAPE;
  const prcr_cache &c = cache->cache;
  // A layer's rows of a sequence, or of a block, have a 32-bit count.
  if (c.paged && static_cast<int64_t>(c.block_size) * n_kv_heads > INT32_MAX) return PRCR_ERR_SHAPE;
  if (c.k == nullptr || c.v == nullptr || cache->k_scale == nullptr || cache->v_scale == nullptr ||
      (c.paged && c.block_table == nullptr))
    return PRCR_ERR_NULL;
  if (!aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(cache->k_scale, 4) || !aligned(cache->v_scale, 4) ||
      (c.paged && !aligned(c.block_table, 4)))
    return PRCR_ERR_ALIGN;
  return PRCR_OK;
}

double cache_rows(const prcr_cache &c, int32_t batch, int32_t n_layers, int32_t n_kv_heads) {
  const double slots = c.paged ? static_cast<double>(c.n_blocks) * c.block_size : static_cast<double>(batch) * c.s_max;
  return slots * n_layers * n_kv_heads;
}

QuantStore store_of(const prcr_quant_cache &cache, int32_t n_layers, int32_t n_kv_heads) {
  const prcr_cache &c = cache.cache;
  QuantStore s{};
  s.k = c.k;
  s.v = c.v;
  s.k_scale = cache.k_scale;
  s.v_scale = cache.v_scale;
  s.block_table = c.block_table;
  s.paged = c.paged;
  s.code = cache.code;
  s.n_layers = n_layers;
  s.n_kv_heads = n_kv_heads;
  s.s_max = c.s_max;
  s.block_size = c.block_size;
  s.max_blocks = c.max_blocks;
  s.n_blocks = c.n_blocks;
  if (c.paged) {
    s.layer_rows = s.layer_scales = static_cast<int64_t>(c.n_blocks) * c.block_size * n_kv_heads;
    s.head_rows = 1;
    s.head_scales = c.block_size;
    s.by_block = Divisor::of(c.block_size);
  } else {
    s.layer_rows = s.layer_scales = static_cast<int64_t>(c.s_max) * n_kv_heads;
    s.head_rows = s.head_scales = c.s_max;
  }
  return s;
}

void set_rope(const prcr_rope &rope, AxisMapId map, QuantWriteParams *p) {
  for (int i = 0; i < rope.head_dim / 2; ++i) {
    const int axis = axis_of_pair(map, i);
    p->on_h |= static_cast<uint64_t>(axis == 1) << i;
    p->on_w |= static_cast<uint64_t>(axis == 2) << i;
    p->inv_freq[i] = std::pow(rope.theta, -(2.0 * i) / rope.head_dim);
  }
}

prcr_status decode_shape(const prcr_quant_cache *cache, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                         int32_t head_dim, int *n_split, size_t *bytes) {
  int64_t capacity = 0;
  const prcr_status st = cache_shape(cache, &capacity);
  if (st != PRCR_OK) return st;
  if (batch < 1 || batch > 65535 || n_kv_heads < 1 || n_kv_heads > 65535 || n_q_heads < 1 || n_q_heads > 65535 ||
      n_q_heads % n_kv_heads != 0 || n_q_heads / n_kv_heads > 8)
    return PRCR_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return PRCR_ERR_UNSUPPORTED;
  *n_split = decode_splits(capacity, batch, n_kv_heads, n_q_heads / n_kv_heads);
  *bytes = static_cast<size_t>(batch) * n_q_heads * *n_split * (head_dim + 2) * sizeof(float);
  return PRCR_OK;
}

}  // namespace

extern "C" {

prcr_status prcr_quant_append(const prcr_rope *rope, const prcr_quant_cache *cache, prcr_dtype dtype, int32_t batch,
                              int32_t n_layers, int32_t n_kv_heads, int32_t layer, const void *raw_k,
                              const void *raw_v, int32_t s_src, const int32_t *pos, const int32_t *n_tokens,
                              const int32_t *cache_start, int32_t *err_flag, hipStream_t stream) {
  AxisMapId map;
  int64_t capacity = 0;
  prcr_status st = check_rope(rope, &map);
  if (st == PRCR_OK) st = check_dtype(dtype);
  if (st == PRCR_OK) st = check_cache(cache, batch, n_layers, n_kv_heads, rope->head_dim, &capacity);
  if (st != PRCR_OK) return st;
  if (raw_k == nullptr || raw_v == nullptr || pos == nullptr || n_tokens == nullptr || cache_start == nullptr)
    return PRCR_ERR_NULL;
  if (layer < 0 || layer >= n_layers || s_src < 1 || static_cast<int64_t>(batch) * s_src > INT32_MAX) return PRCR_ERR_SHAPE;
  if (!aligned(raw_k, 16) || !aligned(raw_v, 16) || !aligned(pos, 4) || !aligned(n_tokens, 4) ||
      !aligned(cache_start, 4) || !aligned(err_flag, 4))
    return PRCR_ERR_ALIGN;
  const prcr_cache &c = cache->cache;
  const double rows = cache_rows(c, batch, n_layers, n_kv_heads), tokens = static_cast<double>(batch) * s_src;
  const double raw = tokens * n_kv_heads * rope->head_dim * elem_bytes(dtype), nb4 = 4.0 * batch;
  const Range written[] = {{c.k, rows * rope->head_dim}, {c.v, rows * rope->head_dim}, {cache->k_scale, rows * 4},
                           {cache->v_scale, rows * 4}};
  const Range read[] = {{raw_k, raw}, {raw_v, raw}, {pos, tokens * 12}, {n_tokens, nb4}, {cache_start, nb4},
                        {c.paged ? c.block_table : nullptr, nb4 * c.max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  QuantWriteParams p{};
  p.to = store_of(*cache, n_layers, n_kv_heads);
  p.k = raw_k;
  p.v = raw_v;
  p.pos = pos;
  p.n_tokens = n_tokens;
  p.start = cache_start;
  p.err = err_flag;
  p.batch = batch;
  p.s_src = s_src;
  p.layer = layer;
  p.n_tok = batch * s_src;
  p.rows = n_kv_heads;
  set_rope(*rope, map, &p);
  return launch_status(launch_quant_append(p, dtype, rope->head_dim, stream));
}

prcr_status prcr_quant_rebind_inject(const prcr_rope *rope, const prcr_mem *mem, const int32_t *sel_off,
                                     const int32_t *sel_idx, int32_t total_k, const double *new_pos,
                                     const prcr_quant_cache *cache, const int32_t *cache_len, int32_t *new_cache_len,
                                     int64_t *slot_mapping, int32_t *err_flag, hipStream_t stream) {
  AxisMapId map;
  int64_t capacity = 0;
  prcr_status st = check_rope(rope, &map);
  if (st != PRCR_OK) return st;
  if (mem == nullptr || mem->k == nullptr || mem->n_visual == nullptr) return PRCR_ERR_NULL;
  const bool key_only = mem->v == nullptr;
  if (key_only && mem->v_slot == nullptr) return PRCR_ERR_NULL;
  if ((st = check_dtype(mem->dtype)) != PRCR_OK) return st;
  if (mem->max_visual < 1 || mem->head_dim != rope->head_dim) return PRCR_ERR_SHAPE;
  if ((st = check_cache(cache, mem->batch, mem->n_layers, mem->n_kv_heads, mem->head_dim, &capacity)) != PRCR_OK) return st;
  if (sel_off == nullptr || cache_len == nullptr || (total_k > 0 && (sel_idx == nullptr || new_pos == nullptr)))
    return PRCR_ERR_NULL;
  if (total_k < 0) return PRCR_ERR_SHAPE;
  if (!aligned(mem->k, 16) || !aligned(mem->v, 16) || !aligned(mem->n_visual, 4) || (key_only && !aligned(mem->v_slot, 4)) ||
      !aligned(sel_off, 4) || !aligned(sel_idx, 4) || !aligned(new_pos, 8) || !aligned(cache_len, 4) ||
      !aligned(new_cache_len, 4) || !aligned(slot_mapping, 8) || !aligned(err_flag, 4))
    return PRCR_ERR_ALIGN;
  const prcr_cache &c = cache->cache;
  const double rows = cache_rows(c, mem->batch, mem->n_layers, mem->n_kv_heads), nb4 = 4.0 * mem->batch;
  const double raw = static_cast<double>(mem->batch) * mem->max_visual * mem->n_layers * mem->n_kv_heads *
                     mem->head_dim * elem_bytes(mem->dtype);
  const Range written[] = {{c.k, rows * mem->head_dim}, {c.v, rows * mem->head_dim}, {cache->k_scale, rows * 4},
                           {cache->v_scale, rows * 4}, {new_cache_len, nb4}, {slot_mapping, 8.0 * total_k}};
  const Range read[] = {{mem->k, raw}, {mem->v, raw}, {mem->n_visual, nb4},
                        {key_only ? mem->v_slot : nullptr, nb4 * mem->max_visual}, {sel_off, nb4 + 4},
                        {sel_idx, 4.0 * total_k}, {new_pos, 24.0 * total_k}, {cache_len, nb4},
                        {c.paged ? c.block_table : nullptr, nb4 * c.max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  QuantWriteParams p{};
  p.to = store_of(*cache, mem->n_layers, mem->n_kv_heads);
  p.k = mem->k;
  p.v = mem->v;
  p.start = cache_len;
  p.sel_off = sel_off;
  p.sel_idx = sel_idx;
  p.n_visual = mem->n_visual;
  p.v_slot = key_only ? mem->v_slot : nullptr;
  p.new_pos = new_pos;
  p.new_len = new_cache_len;
  p.slot_mapping = slot_mapping;
  p.err = err_flag;
  p.batch = mem->batch;
  p.max_visual = mem->max_visual;
  p.n_tok = total_k;
  p.rows = mem->n_layers * mem->n_kv_heads;
  set_rope(*rope, map, &p);
  return launch_status(launch_quant_rebind(p, mem->dtype, mem->head_dim, stream));
}

prcr_status prcr_quant_read(const prcr_quant_cache *cache, prcr_dtype dtype, int32_t batch, int32_t n_layers,
                            int32_t n_kv_heads, int32_t head_dim, int32_t layer, const int32_t *cache_len, void *k,
                            void *v, int32_t s_out, int32_t *err_flag, hipStream_t stream) {
  int64_t capacity = 0;
  prcr_status st = check_dtype(dtype);
  if (st == PRCR_OK) st = check_cache(cache, batch, n_layers, n_kv_heads, head_dim, &capacity);
  if (st != PRCR_OK) return st;
  if (cache_len == nullptr || k == nullptr || v == nullptr) return PRCR_ERR_NULL;
  if (layer < 0 || layer >= n_layers || s_out < 1 || s_out > kMaxSlots) return PRCR_ERR_SHAPE;
  if (!aligned(cache_len, 4) || !aligned(k, 16) || !aligned(v, 16) || !aligned(err_flag, 4)) return PRCR_ERR_ALIGN;
  const prcr_cache &c = cache->cache;
  const double rows = cache_rows(c, batch, n_layers, n_kv_heads), nb4 = 4.0 * batch;
  const double out = static_cast<double>(batch) * n_kv_heads * s_out * head_dim * elem_bytes(dtype);
  const Range written[] = {{k, out}, {v, out}};
  const Range read[] = {{c.k, rows * head_dim}, {c.v, rows * head_dim}, {cache->k_scale, rows * 4},
                        {cache->v_scale, rows * 4}, {cache_len, nb4},
                        {c.paged ? c.block_table : nullptr, nb4 * c.max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  QuantReadParams p{};
  p.from = store_of(*cache, n_layers, n_kv_heads);
  p.k = k;
  p.v = v;
  p.cache_len = cache_len;
  p.err = err_flag;
  p.batch = batch;
  p.layer = layer;
  p.s_out = s_out;
  p.capacity = static_cast<int32_t>(capacity);
  return launch_status(launch_quant_read(p, dtype, head_dim, stream));
}

prcr_status prcr_quant_decode_workspace_size(const prcr_quant_cache *cache, int32_t batch, int32_t n_q_heads,
                                             int32_t n_kv_heads, int32_t head_dim, size_t *bytes) {
  if (bytes == nullptr) return PRCR_ERR_NULL;
  int n_split = 0;
  return decode_shape(cache, batch, n_q_heads, n_kv_heads, head_dim, &n_split, bytes);
}

prcr_status prcr_quant_decode_attention(const prcr_rope *rope, const prcr_quant_cache *cache, prcr_dtype dtype,
                                        int32_t batch, int32_t n_layers, int32_t n_kv_heads, int32_t layer,
                                        const void *q, int32_t n_q_heads, const int32_t *q_pos,
                                        const int32_t *cache_len, float scale, float *out, void *workspace,
                                        size_t workspace_bytes, int32_t *err_flag, hipStream_t stream) {
  AxisMapId map;
  int64_t capacity = 0;
  int n_split = 0;
  size_t need = 0;
  prcr_status st = check_rope(rope, &map);
  if (st == PRCR_OK) st = check_dtype(dtype);
  if (st == PRCR_OK) st = check_cache(cache, batch, n_layers, n_kv_heads, rope->head_dim, &capacity);
  if (st == PRCR_OK) st = decode_shape(cache, batch, n_q_heads, n_kv_heads, rope->head_dim, &n_split, &need);
  if (st != PRCR_OK) return st;
  if (q == nullptr || q_pos == nullptr || cache_len == nullptr || out == nullptr || workspace == nullptr)
    return PRCR_ERR_NULL;
  if (layer < 0 || layer >= n_layers || workspace_bytes < need) return PRCR_ERR_SHAPE;
  if (!std::isfinite(scale) || !std::isfinite(scale * 1.4426950408889634f)) return PRCR_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(q_pos, 4) || !aligned(cache_len, 4) || !aligned(out, 4) || !aligned(workspace, 4) ||
      !aligned(err_flag, 4))
    return PRCR_ERR_ALIGN;
  const prcr_cache &c = cache->cache;
  const double rows = cache_rows(c, batch, n_layers, n_kv_heads), nb4 = 4.0 * batch;
  const double qn = static_cast<double>(batch) * n_q_heads * rope->head_dim;
  const Range written[] = {{out, qn * 4}, {workspace, static_cast<double>(need)}};
  const Range read[] = {{q, qn * elem_bytes(dtype)}, {q_pos, nb4}, {cache_len, nb4}, {c.k, rows * rope->head_dim},
                        {c.v, rows * rope->head_dim}, {cache->k_scale, rows * 4}, {cache->v_scale, rows * 4},
                        {c.paged ? c.block_table : nullptr, nb4 * c.max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  QuantDecodeParams p{};
  p.q = q;
  p.q_pos = q_pos;
  p.cache_len = cache_len;
  p.cache_k = c.k;
  p.cache_v = c.v;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.block_table = c.block_table;
  p.out = out;
  p.ws = static_cast<float *>(workspace);
  p.err = err_flag;
  p.q_f32 = dtype == PRCR_F32;
  p.batch = batch;
  p.n_layers = n_layers;
  p.n_kv_heads = n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.layer = layer;
  p.s_max = c.s_max;
  p.block_size = c.block_size;
  p.max_blocks = c.max_blocks;
  p.n_blocks = c.n_blocks;
  p.block_shift = -1;
  if (c.paged && (c.block_size & (c.block_size - 1)) == 0)
    for (int s = 0; s < 31; ++s)
      if ((1 << s) == c.block_size) p.block_shift = s;
  p.n_split = n_split;
  p.scale = scale;
  for (int i = 0; i < rope->head_dim / 2; ++i) p.inv_freq[i] = std::pow(rope->theta, -(2.0 * i) / rope->head_dim);
  return launch_status(launch_quant_decode(p, cache->code, rope->head_dim, c.paged != 0, stream));
}

}  // extern "C"
