// Eviction: each sequence of more than `budget` slots keeps its first keep_first and its last
// keep_last ones and, of the others, those of the highest score (the sum of the heads'
// weights, in double, rounded to float32; equal scores: the lowest slots; a NaN ranks below every
// number).  Kept slots move, in order, to the front of the cache, in every layer.
//
// Kernel 1, a workgroup per sequence: the scores as integers of the same order, the
// budget-th largest of them by four passes over their bytes, and the list of kept slots.
// Kernel 2, a workgroup per sequence, layer, KV head and operand: the rows, in place.  Slot
// kept[i] >= i, so a workgroup that goes through the rows in order, a batch at a time,
// reading all of a batch before it writes it, overwrites no row that it has yet to read.
// Further workgroups of that launch gather the kept weights and rename the slots of a key-only
// memory's values.  What bounds it is reading and writing the moved rows.
#include <algorithm>

#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kSelect = 1024;                // threads of kernel 1
constexpr int kSelectWaves = kSelect / kWave;
constexpr int kMove = 256;                   // threads of kernel 2
constexpr int kDeep = 4;                     // rows of a batch that a thread has a chunk of
constexpr uint32_t kNowhere = ~0u;           // (a pool's slots are at least 128 bytes each: never so many)

// Order of scores as unsigned integers.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);   // (-0 counts as 0)
  if (x != x) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelect) void select_kernel(const EvictParams p) {
  __shared__ uint32_t s_hist[kSelectWaves][256];
  __shared__ uint32_t s_total[256];
  __shared__ uint32_t s_prefix, s_need;
  __shared__ uint32_t s_more[kSelectWaves], s_equal[kSelectWaves];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int lane = tid & (kWave - 1), wave = tid / kWave;
  const int32_t len = p.cache_len[b];
  const int n = clamp_length(len, p.capacity);
  int32_t *const kept = p.kept + static_cast<int64_t>(b) * p.budget;
  const int n_new = min(n, p.budget);
  // For kernel 2: the kept slots that stay in place at the front; paged, where the others come
  // from and go to.
  int32_t *const first_moved = p.first_moved + b;
  if (len != n && tid == 0 && p.err != nullptr) atomicOr(p.err, PRCR_DERR_CAPACITY);
  __syncthreads();                           // (new_len may be cache_len)
  if (tid == 0) p.new_len[b] = n_new;
  for (int i = n_new + tid; i < p.budget; i += kSelect) kept[i] = -1;
  if (n <= p.budget) {
    for (int i = tid; i < n; i += kSelect) kept[i] = i;
    if (tid == 0) *first_moved = n;
    return;
  }
  uint32_t *const order = reinterpret_cast<uint32_t *>(p.score) + static_cast<int64_t>(b) * p.capacity;
  const float *const w = p.weights + static_cast<int64_t>(b) * p.n_kv_heads * p.capacity;
  for (int j = tid; j < n; j += kSelect) {
    double sum = 0.0;
    for (int h = 0; h < p.n_kv_heads; ++h) sum += static_cast<double>(w[static_cast<int64_t>(h) * p.capacity + j]);
    order[j] = j < p.keep_first || j >= n - p.keep_last ? 0xFFFFFFFFu : order_of(static_cast<float>(sum));
  }
  // The budget-th largest: byte by byte, the bucket in which it lies.  (Each thread reads
  // what it wrote.)
  if (tid == 0) {
    s_prefix = 0u;
    s_need = static_cast<uint32_t>(p.budget);
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < kSelectWaves * 256; i += kSelect) (&s_hist[0][0])[i] = 0u;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    for (int j = tid; j < n; j += kSelect) {
      const uint32_t u = order[j];
      if (shift == 24 || u >> (shift + 8) == prefix) atomicAdd(&s_hist[wave][u >> shift & 255u], 1u);
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t sum = 0u;
      for (int v = 0; v < kSelectWaves; ++v) sum += s_hist[v][tid];
      s_total[tid] = sum;
    }
    __syncthreads();
    if (wave == 0) {
      // Counts from the highest bucket down: lane l has buckets 255 - 4 l .. 252 - 4 l.
      uint32_t c[4], sum = 0u;
      for (int e = 0; e < 4; ++e) sum += c[e] = s_total[255 - 4 * lane - e];
      uint32_t below = sum;                  // inclusive prefix over the lanes
      for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t x = __shfl_up(below, d);
        if (lane >= d) below += x;
      }
      uint32_t above = below - sum;
      const uint32_t need = s_need;
      for (int e = 0; e < 4; ++e) {
        if (above < need && need <= above + c[e]) {
          s_prefix = prefix << 8 | static_cast<uint32_t>(255 - 4 * lane - e);
          s_need = need - above;             // of that bucket
        }
        above += c[e];
      }
    }
    __syncthreads();
  }
  const uint32_t least = s_prefix, equal = s_need;
  // Slots above it, and the first `equal` ones at it, in order.
  uint32_t more0 = 0u, equal0 = 0u;          // of the slots before this round's
  int moved = n;
  for (int j0 = 0; j0 < n; j0 += kSelect) {
    const int j = j0 + tid;
    const uint32_t u = j < n ? order[j] : 0u;
    const bool is_more = j < n && u > least, is_equal = j < n && u == least;
    const unsigned long long mb = __ballot(is_more), eb = __ballot(is_equal);
    if (lane == 0) {
      s_more[wave] = static_cast<uint32_t>(__popcll(mb));
      s_equal[wave] = static_cast<uint32_t>(__popcll(eb));
    }
    __syncthreads();
    const unsigned long long before = (1ull << lane) - 1ull;
    uint32_t m = more0 + __popcll(mb & before), e = equal0 + __popcll(eb & before);
    for (int v = 0; v < kSelectWaves; ++v) {
      m += v < wave ? s_more[v] : 0u;
      e += v < wave ? s_equal[v] : 0u;
      more0 += s_more[v];
      equal0 += s_equal[v];
    }
    if (is_more || (is_equal && e < equal)) {
      const uint32_t at = m + min(e, equal);
      kept[at] = j;
      if (static_cast<int>(at) != j) moved = min(moved, static_cast<int>(at));
    }
    __syncthreads();
  }
  for (int d = 1; d < kWave; d <<= 1) moved = min(moved, __shfl_xor(moved, d));
  if (lane == 0) s_more[wave] = static_cast<uint32_t>(moved);
  __syncthreads();
  for (int v = 0; v < kSelectWaves; ++v) moved = min(moved, static_cast<int>(s_more[v]));
  if (tid == 0) *first_moved = moved;
  if (p.moves == nullptr) return;
  // (The barriers above order the list's writes before these reads of it.)
  bool bad = false;
  auto in_pool = [&](int slot) -> uint32_t {
    const int lb = slot / p.block_size;
    const int32_t blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + lb];
    const bool ok = blk >= 0 && blk < p.n_blocks;
    bad |= !ok;
    return ok ? static_cast<uint32_t>(blk) * static_cast<uint32_t>(p.block_size) +
                    static_cast<uint32_t>(slot - lb * p.block_size) : kNowhere;
  };
  for (int i = moved + tid; i < p.budget; i += kSelect) {
    const uint32_t from = in_pool(kept[i]), to = in_pool(i);
    p.moves[static_cast<int64_t>(b) * p.budget + i] = from == kNowhere || to == kNowhere ? u32x2{kNowhere, kNowhere}
                                                                                         : u32x2{from, to};
  }
  if (bad && p.err != nullptr) atomicOr(p.err, PRCR_DERR_BLOCK);
}

template <bool kPaged>
__global__ __launch_bounds__(kMove) void move_kernel(const EvictParams p, const uint32_t n_move, const Divisor by_heads,
                                                     const Divisor by_layers, const Divisor by_batch) {
  const int tid = threadIdx.x;
  uint32_t id = blockIdx.x;
  if (id >= n_move) {
    // Weights of one sequence and head, then the memories.
    id -= n_move;
    const uint32_t n_heads = p.new_weights != nullptr ? static_cast<uint32_t>(p.batch) * p.n_kv_heads : 0u;
    if (id < n_heads) {
      const int b = static_cast<int>(by_heads.divide(id));
      const int32_t *const kept = p.kept + static_cast<int64_t>(b) * p.budget;
      const float *const from = p.weights + static_cast<int64_t>(id) * p.capacity;
      float *const to = p.new_weights + static_cast<int64_t>(id) * p.capacity;
      const int n = p.new_len[b];
      for (int i = tid; i < p.capacity; i += kMove) to[i] = i < n ? from[kept[i]] : 0.f;
      return;
    }
    const int b = static_cast<int>(id - n_heads);
    const int32_t *const kept = p.kept + static_cast<int64_t>(b) * p.budget;
    const int n = p.new_len[b];
    for (int v = tid; v < p.max_visual; v += kMove) {
      int32_t *const slot = p.v_slot + static_cast<int64_t>(b) * p.max_visual + v;
      const int32_t old = *slot;
      int lo = 0, hi = n;                    // the first kept slot at or above it
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (kept[mid] < old) lo = mid + 1; else hi = mid;
      }
      *slot = old >= 0 && lo < n && kept[lo] == old ? lo : -1;
    }
    return;
  }
  const uint32_t by_head = by_heads.divide(id);
  const int kvh = static_cast<int>(id - by_head * static_cast<uint32_t>(p.n_kv_heads));
  const uint32_t by_layer = by_layers.divide(by_head);
  const int layer = static_cast<int>(by_head - by_layer * static_cast<uint32_t>(p.n_layers));
  const uint32_t operand = by_batch.divide(by_layer);
  const int b = static_cast<int>(by_layer - operand * static_cast<uint32_t>(p.batch));
  const int n = p.new_len[b], i0 = p.first_moved[b];
  if (i0 >= n) return;
  const int chunks = p.row_bytes / 16;       // a power of two, at most 32
  const int r = tid / chunks, step = kMove / chunks;
  // Slot 0's row of this layer (paged: the pool's) and head, and the bytes from a slot to the next.
  const int64_t base = kPaged ? static_cast<int64_t>(layer) * p.n_blocks * p.block_size * p.n_kv_heads + kvh
                              : ((static_cast<int64_t>(b) * p.n_layers + layer) * p.n_kv_heads + kvh) * p.s_max;
  char *const rows = static_cast<char *>(operand != 0 ? p.cache_v : p.cache_k) + base * p.row_bytes +
                     (tid & (chunks - 1)) * 16;
  const uint64_t slot_bytes = static_cast<uint64_t>(p.row_bytes) * (kPaged ? p.n_kv_heads : 1);
  const int32_t *const kept = p.kept + static_cast<int64_t>(b) * p.budget;
  const u32x2 *const moves = kPaged ? p.moves + static_cast<int64_t>(b) * p.budget : nullptr;
  struct Batch {
    u32x4 x[kDeep];
    u32x2 slots[kDeep];                      // from, to
  };
  auto look_up = [&](int first, Batch &d) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int i = first + u * step + r;
      d.slots[u] = u32x2{kNowhere, kNowhere};
      if (i < n) d.slots[u] = kPaged ? moves[i] : u32x2{static_cast<uint32_t>(kept[i]), static_cast<uint32_t>(i)};
    }
  };
  auto load = [&](Batch &d) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
      if (d.slots[u][0] != kNowhere) d.x[u] = load_nt(rows + d.slots[u][0] * slot_bytes);
  };
  auto store = [&](Batch &d) {
    // Every thread's share of the batch is in registers before one of it is written.
#pragma unroll
    for (int u = 0; u < kDeep; ++u) asm volatile("" : "+v"(d.x[u]));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
      if (d.slots[u][1] != kNowhere) store_nt(rows + d.slots[u][1] * slot_bytes, d.x[u]);
  };
  // The next batch is on its way while one is written: it reads slots from its own first row
  // on, which lie behind all that is written before it.
  const int batch = kDeep * step;
  Batch one, two;
  look_up(i0, one);
  load(one);
  look_up(i0 + batch, two);
  for (int i = i0; i < n; i += 2 * batch) {
    load(two);
    store(one);
    look_up(i + 2 * batch, one);
    load(one);
    store(two);
    look_up(i + 3 * batch, two);
  }
}

}  // namespace

hipError_t launch_evict(const EvictParams &p, bool paged, hipStream_t stream) {
  const int64_t n_move = int64_t{2} * p.batch * p.n_layers * p.n_kv_heads;
  const int64_t blocks = n_move + (p.new_weights != nullptr ? int64_t{1} * p.batch * p.n_kv_heads : 0) +
                         (p.v_slot != nullptr ? p.batch : 0);
  if (blocks > INT32_MAX || !grid_fits(blocks, kMove) || !grid_fits(p.batch, kSelect)) return hipErrorInvalidConfiguration;
  select_kernel<<<static_cast<unsigned>(p.batch), kSelect, 0, stream>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const Divisor heads = Divisor::of(p.n_kv_heads), layers = Divisor::of(p.n_layers), batch = Divisor::of(p.batch);
  const uint32_t moves = static_cast<uint32_t>(n_move);
  if (paged)
    move_kernel<true><<<static_cast<unsigned>(blocks), kMove, 0, stream>>>(p, moves, heads, layers, batch);
  else
    move_kernel<false><<<static_cast<unsigned>(blocks), kMove, 0, stream>>>(p, moves, heads, layers, batch);
  return hipGetLastError();
}

}  // namespace prcr
