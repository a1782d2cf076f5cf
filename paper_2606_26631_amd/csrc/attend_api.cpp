// extern "C" entry points of the operators on several tokens per sequence (chunk
// attention, the keys' weights, eviction): structural validation on the host, then the
// launches on the caller's stream.  No entry point allocates or keeps state.
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "attend.h"

using namespace prcr;

namespace {

constexpr int64_t kMaxSlots = int64_t{1} << 30;    // cache capacity per sequence, rows per KV head, and budget

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

int elem_bytes(prcr_dtype d) { return d == PRCR_F32 ? 4 : 2; }

prcr_status check_rope(const prcr_rope *rope) {
  if (rope == nullptr) return PRCR_ERR_NULL;
  const int d = rope->head_dim;
  if (d < 2 || d % 2 != 0 || d / 2 > kMaxPairs) return PRCR_ERR_SHAPE;
  for (int a = 0; a < 3; ++a)
    if (rope->section[a] < 0) return PRCR_ERR_SHAPE;
  if (static_cast<int64_t>(rope->section[0]) + rope->section[1] + rope->section[2] != d / 2) return PRCR_ERR_SHAPE;
  if (rope->interleaved != 0 && rope->interleaved != 1) return PRCR_ERR_SHAPE;
  if (!(rope->theta > 0.0) || !std::isfinite(rope->theta)) return PRCR_ERR_SHAPE;
  return PRCR_OK;
}

// Layout flag and geometry of a cache; the slots a sequence has.
prcr_status cache_shape(const prcr_cache *cache, int64_t *capacity) {
  if (cache == nullptr) return PRCR_ERR_NULL;
  if (cache->paged != 0 && cache->paged != 1) return PRCR_ERR_SHAPE;
  if (cache->paged) {
    if (cache->block_size < 1 || cache->max_blocks < 1 || cache->n_blocks < 1) return PRCR_ERR_SHAPE;
    *capacity = static_cast<int64_t>(cache->max_blocks) * cache->block_size;
  } else {
    if (cache->s_max < 1) return PRCR_ERR_SHAPE;
    *capacity = cache->s_max;
  }
  return *capacity > kMaxSlots ? PRCR_ERR_SHAPE : PRCR_OK;
}

prcr_status check_cache(const prcr_cache *cache, int64_t *capacity) {
  const prcr_status st = cache_shape(cache, capacity);
  if (st != PRCR_OK) return st;
  if (cache->k == nullptr || cache->v == nullptr || (cache->paged && cache->block_table == nullptr)) return PRCR_ERR_NULL;
  if (!aligned(cache->k, 16) || !aligned(cache->v, 16) || (cache->paged && !aligned(cache->block_table, 4)))
    return PRCR_ERR_ALIGN;
  return PRCR_OK;
}

prcr_status check_heads(int32_t batch, int32_t n_kv_heads, int32_t head_dim) {
  if (batch < 1 || batch > 65535 || n_kv_heads < 1 || n_kv_heads > 65535) return PRCR_ERR_SHAPE;
  return head_dim == 64 || head_dim == 128 ? PRCR_OK : PRCR_ERR_UNSUPPORTED;
}

prcr_status check_rows(int32_t total_q, int32_t n_q_heads, int32_t n_kv_heads) {
  if (total_q < 0 || n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % n_kv_heads != 0) return PRCR_ERR_SHAPE;
  return static_cast<int64_t>(total_q) * n_q_heads > kMaxSlots ? PRCR_ERR_SHAPE : PRCR_OK;
}

double cache_bytes(const prcr_cache &c, int32_t batch, int32_t n_layers, int32_t n_kv_heads, double row_bytes) {
  const double slots = c.paged ? static_cast<double>(c.n_blocks) * c.block_size : static_cast<double>(batch) * c.s_max;
  return slots * n_layers * n_kv_heads * row_bytes;
}

// Checks and parameter block that chunk attention and the keys' weights share.
prcr_status prepare(const prcr_rope *rope, const prcr_cache *cache, prcr_dtype dtype, int32_t batch, int32_t n_layers,
                    int32_t n_kv_heads, int32_t layer, const void *q, int32_t n_q_heads, const int32_t *q_off,
                    const int32_t *q_len, int32_t total_q, const int32_t *q_pos, const int32_t *cache_len, float scale,
                    void *workspace, int32_t *err_flag, AttendParams *out) {
  prcr_status st = check_rope(rope);
  if (st != PRCR_OK) return st;
  if (dtype != PRCR_F32 && dtype != PRCR_BF16) return PRCR_ERR_DTYPE;
  if ((st = check_heads(batch, n_kv_heads, rope->head_dim)) != PRCR_OK) return st;
  if ((st = check_rows(total_q, n_q_heads, n_kv_heads)) != PRCR_OK) return st;
  int64_t capacity = 0;
  if ((st = check_cache(cache, &capacity)) != PRCR_OK) return st;
  if (q_off == nullptr || cache_len == nullptr) return PRCR_ERR_NULL;
  if (total_q > 0 && (q == nullptr || q_pos == nullptr)) return PRCR_ERR_NULL;
  if (n_layers < 1 || layer < 0 || layer >= n_layers) return PRCR_ERR_SHAPE;
  if (!std::isfinite(scale) || !std::isfinite(scale * 1.4426950408889634f)) return PRCR_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(q_off, 4) || !aligned(q_len, 4) || !aligned(q_pos, 4) || !aligned(cache_len, 4) ||
      !aligned(workspace, 16) || !aligned(err_flag, 4))
    return PRCR_ERR_ALIGN;
  const AxisMapId map = axis_map_id(*rope);
  if (map == AxisMapId::kUnsupported) return PRCR_ERR_UNSUPPORTED;
  AttendParams &p = *out;
  p = AttendParams{};
  p.q = q;
  p.rotated = workspace;
  p.q_off = q_off;
  p.q_len = q_len;
  p.q_pos = q_pos;
  p.cache_len = cache_len;
  p.cache_k = cache->k;
  p.cache_v = cache->v;
  p.block_table = cache->block_table;
  p.err = err_flag;
  p.total_q = total_q;
  p.batch = batch;
  p.n_layers = n_layers;
  p.n_kv_heads = n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.group = n_q_heads / n_kv_heads;
  p.layer = layer;
  p.s_max = cache->s_max;
  p.block_size = cache->block_size;
  p.max_blocks = cache->max_blocks;
  p.n_blocks = cache->n_blocks;
  p.block_shift = -1;
  if (cache->paged && (cache->block_size & (cache->block_size - 1)) == 0)
    for (int s = 0; s < 31; ++s)
      if ((1 << s) == cache->block_size) p.block_shift = s;
  p.capacity = static_cast<int32_t>(capacity);
  p.negate = scale < 0.f;
  p.scale2 = static_cast<float>(std::fabs(static_cast<double>(scale)) * 1.4426950408889634);
  p.by_group = Divisor::of(p.group);
  p.by_heads = Divisor::of(n_kv_heads);
  for (int i = 0; i < rope->head_dim / 2; ++i) {
    p.axis[i] = static_cast<int8_t>(axis_of_pair(map, i));
    p.inv_freq[i] = std::pow(rope->theta, -(2.0 * i) / rope->head_dim);
  }
  return PRCR_OK;
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

}  // namespace

extern "C" {

prcr_status prcr_chunk_workspace_size(const prcr_cache *cache, int32_t batch, int32_t total_q, int32_t n_q_heads,
                                      int32_t n_kv_heads, int32_t head_dim, size_t *bytes) {
  if (bytes == nullptr) return PRCR_ERR_NULL;
  int64_t capacity = 0;
  prcr_status st = check_heads(batch, n_kv_heads, head_dim);
  if (st == PRCR_OK) st = check_rows(total_q, n_q_heads, n_kv_heads);
  if (st == PRCR_OK) st = cache_shape(cache, &capacity);
  if (st != PRCR_OK) return st;
  *bytes = plan_chunk(capacity, batch, total_q, n_q_heads, n_kv_heads, head_dim).bytes;
  return PRCR_OK;
}

prcr_status prcr_chunk_attention(const prcr_rope *rope, const prcr_cache *cache, prcr_dtype dtype, int32_t batch,
                                 int32_t n_layers, int32_t n_kv_heads, int32_t layer, const void *q, int32_t n_q_heads,
                                 const int32_t *q_off, const int32_t *q_len, int32_t total_q, const int32_t *q_pos,
                                 const int32_t *cache_len, float scale, void *out, float *lse, void *workspace,
                                 size_t workspace_bytes, int32_t *err_flag, hipStream_t stream) {
  AttendParams p;
  const prcr_status st = prepare(rope, cache, dtype, batch, n_layers, n_kv_heads, layer, q, n_q_heads, q_off, q_len,
                                 total_q, q_pos, cache_len, scale, workspace, err_flag, &p);
  if (st != PRCR_OK) return st;
  if (total_q == 0) return PRCR_OK;
  if (out == nullptr) return PRCR_ERR_NULL;
  const ChunkPlan plan = plan_chunk(p.capacity, batch, total_q, n_q_heads, n_kv_heads, rope->head_dim);
  if (plan.bytes > 0 && workspace == nullptr) return PRCR_ERR_NULL;
  if (workspace_bytes < plan.bytes) return PRCR_ERR_SHAPE;
  if (!aligned(out, 16) || !aligned(lse, 4)) return PRCR_ERR_ALIGN;
  const double row_bytes = static_cast<double>(rope->head_dim) * elem_bytes(dtype), rows = static_cast<double>(total_q) * n_q_heads;
  const double all = cache_bytes(*cache, batch, n_layers, n_kv_heads, row_bytes);
  const Range written[] = {{out, rows * row_bytes}, {lse, rows * 4}, {workspace, static_cast<double>(plan.bytes)}};
  const Range read[] = {{q, rows * row_bytes}, {q_off, (batch + 1) * 4.0}, {q_len, batch * 4.0}, {q_pos, total_q * 12.0},
                        {cache_len, batch * 4.0}, {cache->k, all}, {cache->v, all},
                        {cache->paged ? cache->block_table : nullptr, 4.0 * batch * cache->max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  p.out = out;
  p.lse = lse;
  p.part = static_cast<float *>(workspace);
  return launch_status(launch_chunk(p, plan, dtype, rope->head_dim, cache->paged != 0, stream));
}

prcr_status prcr_key_weights_workspace_size(const prcr_cache *cache, prcr_dtype dtype, int32_t batch, int32_t total_q,
                                            int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t window,
                                            size_t *bytes) {
  if (bytes == nullptr) return PRCR_ERR_NULL;
  if (dtype != PRCR_F32 && dtype != PRCR_BF16) return PRCR_ERR_DTYPE;
  int64_t capacity = 0;
  prcr_status st = check_heads(batch, n_kv_heads, head_dim);
  if (st == PRCR_OK) st = check_rows(total_q, n_q_heads, n_kv_heads);
  if (st == PRCR_OK) st = cache_shape(cache, &capacity);
  if (st == PRCR_OK && window < 0) st = PRCR_ERR_SHAPE;
  if (st != PRCR_OK) return st;
  *bytes = plan_key_weights(capacity, batch, total_q, n_q_heads, n_kv_heads, head_dim, window, dtype).bytes;
  return PRCR_OK;
}

prcr_status prcr_key_weights(const prcr_rope *rope, const prcr_cache *cache, prcr_dtype dtype, int32_t batch,
                             int32_t n_layers, int32_t n_kv_heads, int32_t layer, const void *q, int32_t n_q_heads,
                             const int32_t *q_off, const int32_t *q_len, int32_t total_q, const int32_t *q_pos,
                             const int32_t *cache_len, const float *lse, int32_t window, float scale,
                             int32_t accumulate, float *weights, void *workspace, size_t workspace_bytes,
                             int32_t *err_flag, hipStream_t stream) {
  AttendParams p;
  const prcr_status st = prepare(rope, cache, dtype, batch, n_layers, n_kv_heads, layer, q, n_q_heads, q_off, q_len,
                                 total_q, q_pos, cache_len, scale, workspace, err_flag, &p);
  if (st != PRCR_OK) return st;
  if (weights == nullptr || (total_q > 0 && (lse == nullptr || workspace == nullptr))) return PRCR_ERR_NULL;
  if (window < 0) return PRCR_ERR_SHAPE;
  const double row_bytes = static_cast<double>(rope->head_dim) * elem_bytes(dtype), rows = static_cast<double>(total_q) * n_q_heads;
  const WeightsPlan plan = plan_key_weights(p.capacity, batch, total_q, n_q_heads, n_kv_heads, rope->head_dim, window, dtype);
  if (workspace_bytes < plan.bytes) return PRCR_ERR_SHAPE;
  if (!aligned(weights, 4) || !aligned(lse, 4)) return PRCR_ERR_ALIGN;
  const double all = cache_bytes(*cache, batch, n_layers, n_kv_heads, row_bytes);
  const Range written[] = {{weights, 4.0 * batch * n_kv_heads * p.capacity}, {workspace, static_cast<double>(plan.bytes)}};
  const Range read[] = {{q, rows * row_bytes}, {lse, rows * 4}, {q_off, (batch + 1) * 4.0}, {q_len, batch * 4.0},
                        {q_pos, total_q * 12.0}, {cache_len, batch * 4.0}, {cache->k, all}, {cache->v, all},
                        {cache->paged ? cache->block_table : nullptr, 4.0 * batch * cache->max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  p.lse = const_cast<float *>(lse);
  p.weights = weights;
  p.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan.rotated_bytes);
  p.window = window;
  p.accumulate = accumulate != 0;
  if (total_q == 0 && p.accumulate) return PRCR_OK;   // no row gives any weight
  if (total_q > 0 || err_flag != nullptr) {
    const prcr_status first = launch_status(total_q > 0 ? launch_rotate(p, dtype, rope->head_dim, stream)
                                                        : launch_report(p, stream));
    if (first != PRCR_OK) return first;
  }
  return launch_status(launch_key_weights(p, plan, dtype, rope->head_dim, cache->paged != 0, stream));
}

prcr_status prcr_evict_workspace_size(const prcr_cache *cache, int32_t batch, int32_t budget, size_t *bytes) {
  if (bytes == nullptr) return PRCR_ERR_NULL;
  int64_t capacity = 0;
  prcr_status st = check_heads(batch, 1, 64);
  if (st == PRCR_OK) st = cache_shape(cache, &capacity);
  if (st == PRCR_OK && (budget < 1 || budget > kMaxSlots)) st = PRCR_ERR_SHAPE;
  if (st != PRCR_OK) return st;
  // Paged: a kept slot's two places; then the scores; then the first slots that move.
  *bytes = static_cast<size_t>(batch) * ((cache->paged ? static_cast<size_t>(budget) * 8 : 0) +
                                         (static_cast<size_t>(capacity) + 1) * 4);
  return PRCR_OK;
}

prcr_status prcr_evict(const prcr_cache *cache, prcr_dtype dtype, int32_t batch, int32_t n_layers, int32_t n_kv_heads,
                       int32_t head_dim, const int32_t *cache_len, const float *weights, int32_t budget,
                       int32_t keep_first, int32_t keep_last, int32_t *new_cache_len, int32_t *kept,
                       float *new_weights, const prcr_mem *mem, void *workspace, size_t workspace_bytes,
                       int32_t *err_flag, hipStream_t stream) {
  if (dtype != PRCR_F32 && dtype != PRCR_BF16) return PRCR_ERR_DTYPE;
  prcr_status st = check_heads(batch, n_kv_heads, head_dim);
  if (st != PRCR_OK) return st;
  int64_t capacity = 0;
  if ((st = check_cache(cache, &capacity)) != PRCR_OK) return st;
  if (cache_len == nullptr || weights == nullptr || new_cache_len == nullptr || kept == nullptr || workspace == nullptr)
    return PRCR_ERR_NULL;
  if (n_layers < 1 || budget < 1 || keep_first < 0 || keep_last < 0 ||
      static_cast<int64_t>(keep_first) + keep_last > budget)
    return PRCR_ERR_SHAPE;
  size_t need = 0;
  if ((st = prcr_evict_workspace_size(cache, batch, budget, &need)) != PRCR_OK) return st;
  if (workspace_bytes < need) return PRCR_ERR_SHAPE;
  // Only a key-only memory names cache slots.
  const bool rename = mem != nullptr && mem->v == nullptr;
  if (rename) {
    if (mem->v_slot == nullptr) return PRCR_ERR_NULL;
    if (mem->batch != batch || mem->max_visual < 1 || mem->max_visual > kMaxSlots) return PRCR_ERR_SHAPE;
    if (!aligned(mem->v_slot, 4)) return PRCR_ERR_ALIGN;
  }
  if (!aligned(cache_len, 4) || !aligned(weights, 4) || !aligned(new_cache_len, 4) || !aligned(kept, 4) ||
      !aligned(new_weights, 4) || !aligned(workspace, 8) || !aligned(err_flag, 4))
    return PRCR_ERR_ALIGN;
  const double all = cache_bytes(*cache, batch, n_layers, n_kv_heads, static_cast<double>(head_dim) * elem_bytes(dtype));
  const double w = 4.0 * batch * n_kv_heads * static_cast<double>(capacity), nb4 = batch * 4.0;
  const Range written[] = {{cache->k, all}, {cache->v, all}, {new_cache_len, nb4}, {kept, nb4 * budget}, {new_weights, w},
                           {rename ? mem->v_slot : nullptr, rename ? nb4 * mem->max_visual : 0.0},
                           {workspace, static_cast<double>(need)}};
  // (The new lengths may be written in place: a workgroup reads its own one first.)
  const Range read[] = {{new_cache_len == cache_len ? nullptr : cache_len, nb4}, {weights, w},
                        {cache->paged ? cache->block_table : nullptr, nb4 * cache->max_blocks}};
  if (aliases(written, read)) return PRCR_ERR_ALIAS;
  EvictParams p{};
  p.cache_len = cache_len;
  p.weights = weights;
  p.cache_k = cache->k;
  p.cache_v = cache->v;
  p.block_table = cache->block_table;
  p.new_len = new_cache_len;
  p.kept = kept;
  p.new_weights = new_weights;
  p.v_slot = rename ? mem->v_slot : nullptr;
  char *const scores = static_cast<char *>(workspace) + (cache->paged ? static_cast<size_t>(batch) * budget * 8 : 0);
  p.moves = cache->paged ? static_cast<decltype(p.moves)>(workspace) : nullptr;
  p.score = reinterpret_cast<float *>(scores);
  p.first_moved = reinterpret_cast<int32_t *>(p.score + static_cast<int64_t>(batch) * capacity);
  p.err = err_flag;
  p.batch = batch;
  p.n_layers = n_layers;
  p.n_kv_heads = n_kv_heads;
  p.row_bytes = head_dim * elem_bytes(dtype);
  p.s_max = cache->s_max;
  p.block_size = cache->block_size;
  p.max_blocks = cache->max_blocks;
  p.n_blocks = cache->n_blocks;
  p.capacity = static_cast<int32_t>(capacity);
  p.budget = budget;
  p.keep_first = keep_first;
  p.keep_last = keep_last;
  p.max_visual = rename ? mem->max_visual : 0;
  return launch_status(launch_evict(p, cache->paged != 0, stream));
}

}  // extern "C"
