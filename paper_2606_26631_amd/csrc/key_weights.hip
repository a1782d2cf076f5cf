// The weight each cached key received from the last tokens: for every sequence b, KV head h
// and slot j,
//   w[b][h][j] (+)= sum over the rows that see j, and the heads of group h, of exp(s_j - lse),
// s_j and lse as chunk attention has them.
//
// A workgroup takes a stretch of keys of one sequence and KV head, 32 kBlocks keys a wave, in
// registers, and runs through the rows that see them, a tile at a time, which all its waves
// read from LDS, the next tile's loads in flight.  The scores are formed as
// Q (32 rows) x K^T (32 keys), so that a lane holds 16 rows' scores of one key and adds
// their weights in its own registers: no other lane's, no atomics, a fixed order.  Where
// that makes few workgroups, the rows are shared out over several, whose sums a second
// kernel adds in order.
//
// What bounds it: of few rows, reading the keys (one token of 32 sequences of 3,500 slots, 8 heads of
// 128: 230 MB in 45 us, 5.1 TB/s); of many, an exponential and a sum per score beside the products
// (4 prompts of 2,560 tokens, 32 heads: 160 us, 0.67 PF of products).  In between, a workgroup's start
// counts: it waits for its stretch of keys before the first product, and has few row tiles for them.
#include <algorithm>
#include <type_traits>

#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;

__device__ __forceinline__ void load_to_lds(const char *from, char *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

template <typename T, int D, bool kPaged, int kBlocks>
__global__ __launch_bounds__(kThreads, 2) void key_weights_kernel(const AttendParams p) {
  constexpr bool kHalf = sizeof(T) == 2;
  constexpr int kRowBytes = D * static_cast<int>(sizeof(T));
  constexpr int kChunks = kRowBytes / 16;
  constexpr int kRowsPerLoad = kWave / kChunks;
  constexpr int kTileBlocks = kHalf ? 2 : 1;                // 32 rows each
  constexpr int kRows = 32 * kTileBlocks;                   // of a tile
  constexpr int kMine = kRows / kRowsPerLoad / kWaves;      // loads of a tile per wave
  constexpr int kQ = kHalf ? D / 16 : D / 8;
  constexpr int kKeys = kWaves * 32 * kBlocks;
  constexpr int kBytes = kRows * kRowBytes;
  constexpr int kKeyBytes = kWaves * 32 * kRowBytes;
  static_assert(kMine >= 1, "a row tile is at least a load per wave");
  // Three tiles of rows.  The keys pass through there too: bf16, through the places of the
  // second and third tile while the first one comes; float32, whose keys take more, before it.
  constexpr bool kEarly = kHalf;
  constexpr int kKeysAt = kEarly ? kBytes : 0;
  __shared__ __align__(1024) char s_rows[3 * kBytes > kKeysAt + kKeyBytes ? 3 * kBytes : kKeysAt + kKeyBytes];
  __shared__ __align__(16) float s_lse[2][kRows];
  __shared__ __align__(16) int s_limit[2][kRows];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane & 31, half = lane / 32;
  const uint32_t id = blockIdx.x;
  const uint32_t by_head = p.by_heads.divide(id);
  const int kvh = static_cast<int>(id - by_head * static_cast<uint32_t>(p.n_kv_heads));
  const uint32_t by_part = p.by_split.divide(by_head);
  const int part = static_cast<int>(by_head - by_part * static_cast<uint32_t>(p.n_split));
  const int b = static_cast<int>(p.by_slot.divide(by_part));       // (n_slots: key stretches per sequence)
  const int k0 = (static_cast<int>(by_part) - b * p.n_slots) * kKeys;
  const int32_t len = clamp_length(p.cache_len[b], p.capacity);
  const int64_t head = static_cast<int64_t>(b) * p.n_kv_heads + kvh;
  float *const weights = p.weights + head * p.capacity;
  if (k0 >= len) {
    if (!p.accumulate && p.n_split == 1)
      for (int j = k0 + threadIdx.x; j < min(k0 + kKeys, p.capacity); j += kThreads) weights[j] = 0.f;
    return;
  }
  const Rows rows = rows_of(p, b);
  const int G = p.group, first = len - rows.n;
  const int from = max(p.window > 0 ? max(rows.n - p.window, 0) : 0, k0 - first);   // first token that counts
  // This workgroup's rows: a share of the tiles that see some of the stretch.
  const int all0 = min(from, rows.n) * G, all1 = rows.n * G;
  const int per = ((all1 - all0 + kRows - 1) / kRows + p.n_split - 1) / p.n_split * kRows;
  const int row0 = min(all0 + part * per, all1), n_rows = min(row0 + per, all1);

  const int in_load = lane / kChunks, chunk = lane % kChunks;
  const int sw = l32 & (kChunks - 1);
  auto token_of = [&](int r) -> int { return static_cast<int>(p.by_group.divide(static_cast<uint32_t>(r))); };
  auto row_index = [&](int r, int token) -> int64_t {
    return (static_cast<int64_t>(rows.start) + token) * p.n_q_heads + kvh * G + (r - token * G);
  };
  auto load_rows = [&](int r0, char *to) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int load = i * kWaves + wave;
      const int at = load * kRowsPerLoad + in_load;
      const int r = min(r0 + at, n_rows - 1);
      load_to_lds(static_cast<const char *>(p.rotated) + row_index(r, token_of(r)) * kRowBytes +
                      (chunk ^ (at & (kChunks - 1))) * 16, to + load * 1024);
    }
  };
  // Of row `lane` of a tile (every wave has them): its log-sum-exp, and the last slot it sees.
  constexpr int kPast = INT32_MIN;           // (a row past the last one)
  float lse = 0.f;
  int limit = kPast;
  auto load_lse = [&](int r0) {
    const int r = r0 + lane % kRows, at = min(r, n_rows - 1);
    const int token = token_of(at);
    limit = r < n_rows ? first + token : kPast;
    lse = p.lse[row_index(at, token)];
  };
  // What is taken from the rows' scores (base 2), and the last slots, to LDS.  Rows that see no slot,
  // or have an lse of -infinity, give no weight, whatever their scores are: to the mask they see
  // none.  Whether there is one, and the tile needs the mask for it.  (Rows past the last one, whose
  // scores are that one's again, need none: nothing is left of a number less the largest one, and
  // what is no number, or infinite, has come from the last row already.)
  auto keep_lse = [&](int to) -> bool {
    const bool none = limit < 0 || lse == -__builtin_inff();
    if (threadIdx.x < kRows) {
      s_lse[to][threadIdx.x] = none ? FLT_MAX : lse * 1.44269504088896341f;
      s_limit[to][threadIdx.x] = none ? -1 : limit;
    }
    return __any(none && limit != kPast);
  };

  if (row0 < n_rows) {
    load_lse(row0);
    if (kEarly) load_rows(row0, s_rows);
  }

  // The wave's keys, whole rows through LDS (in the operand's layout a load would read
  // half of each of 32 rows' cache lines).  bf16: of product i, elements 16 i + 8 half + 0..7;
  // float32: the lane's half of the row.
  const int kw = k0 + wave * 32 * kBlocks;
  u32x4 k[kBlocks][kQ];
  bool live[kBlocks];
  bool bad_block = false;
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb) {
    const int mine = kw + 32 * kb + l32;
    const int j = min(mine, len - 1);
    live[kb] = mine < len;
    uint32_t slot = static_cast<uint32_t>(j);
    if constexpr (kPaged) {
      const int lb = p.block_shift >= 0 ? j >> p.block_shift : j / p.block_size;
      const int32_t blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + lb];
      const bool ok = blk >= 0 && blk < p.n_blocks;
      bad_block |= live[kb] && !ok;
      live[kb] = live[kb] && ok;
      // (A pool's slots are at least 128 bytes each: below 2^32 of them.)
      slot = ok ? static_cast<uint32_t>(blk) * static_cast<uint32_t>(p.block_size) +
                      static_cast<uint32_t>(j - lb * p.block_size) : 0u;
    }
    const int64_t base = kPaged ? static_cast<int64_t>(p.layer) * p.n_blocks * p.block_size * p.n_kv_heads + kvh
                                : ((static_cast<int64_t>(b) * p.n_layers + p.layer) * p.n_kv_heads + kvh) * p.s_max;
    const uint32_t step = kPaged ? static_cast<uint32_t>(p.n_kv_heads) : 1u;
    char *const to = s_rows + kKeysAt + wave * 32 * kRowBytes;
#pragma unroll
    for (int i = 0; i < 32 / kRowsPerLoad; ++i) {
      const int at = i * kRowsPerLoad + in_load;
      const uint32_t row = static_cast<uint32_t>(__shfl(static_cast<int>(slot), at));
      load_to_lds(static_cast<const char *>(p.cache_k) +
                      (base + static_cast<int64_t>(static_cast<uint64_t>(row) * step)) * kRowBytes +
                      (chunk ^ (at & (kChunks - 1))) * 16, to + i * 1024);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (a wave reads only what it loaded)
#pragma unroll
    for (int i = 0; i < kQ; ++i)
      k[kb][i] = *reinterpret_cast<const u32x4 *>(to + l32 * kRowBytes + ((kHalf ? 2 * i + half : half * kQ + i) ^ sw) * 16);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (before the next rows, or the tiles, come there)
  }
  if (kPaged && p.err != nullptr && __any(bad_block) && lane == 0) atomicOr(p.err, PRCR_DERR_BLOCK);
  __syncthreads();

  double w[kBlocks] = {};                    // (the first keys add up every row there is: float32 lost 1e-6 of 10,000)
  if (!kEarly && row0 < n_rows) load_rows(row0, s_rows);
  int buf = 0, place = 0;                    // of the present tile, among two and three
  bool none = row0 < n_rows && keep_lse(0);  // a row of the present tile gives no weight
  auto add = [&](auto is_masked) {
    constexpr bool kMasked = decltype(is_masked)::value;
#pragma unroll
    for (int rb = 0; rb < kTileBlocks; ++rb) {
      const char *const qrow = s_rows + place * kBytes + (32 * rb + l32) * kRowBytes;
      f32x16 s[kBlocks];
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        if constexpr (kHalf) {
          const bf16x8 q = *reinterpret_cast<const bf16x8 *>(qrow + ((2 * i + half) ^ sw) * 16);
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb)
            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, __builtin_bit_cast(bf16x8, k[kb][i]), s[kb], 0, 0, 0);
        } else {
          const f32x4 q = *reinterpret_cast<const f32x4 *>(qrow + ((half * kQ + i) ^ sw) * 16);
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb) {
            const f32x4 x = __builtin_bit_cast(f32x4, k[kb][i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[e], x[e], s[kb], 0, 0, 0);
          }
        }
      }
      // The lane's rows 8 (i / 4) + 4 half + i % 4.
      float sum[kBlocks] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 32 * rb + 8 * i + 4 * half;
        const f32x4 off = *reinterpret_cast<const f32x4 *>(&s_lse[buf][at]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int last = kMasked ? s_limit[buf][at + e] : 0;
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb) {
            // (The factor log2 e is in scale2 and in off, in each with a rounding of its own.)
            const float x = exp2_hw(fmaf(s[kb][4 * i + e], p.scale2, -off[e]));
            sum[kb] += !kMasked || kw + 32 * kb + l32 <= last ? x : 0.f;
          }
        }
      }
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) w[kb] += static_cast<double>(sum[kb]);
    }
  };
  for (int r0 = row0; r0 < n_rows; r0 += kRows) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const bool more = r0 + kRows < n_rows;
    const int next = place == 2 ? 0 : place + 1;
    if (more) {
      load_rows(r0 + kRows, s_rows + next * kBytes);
      load_lse(r0 + kRows);
    }
    // Rows that all see the whole stretch need no mask.
    if (none || first + token_of(r0) < k0 + kKeys - 1)
      add(std::true_type{});
    else
      add(std::false_type{});
    if (more) none = keep_lse(buf ^ 1);
    buf ^= 1;
    place = next;
  }
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb) {
    const float sum = static_cast<float>(w[kb] + __shfl_xor(w[kb], 32));
    const int j = kw + 32 * kb + l32;
    if (half != 0 || j >= p.capacity) continue;
    if (p.n_split > 1)
      p.part[(static_cast<int64_t>(part) * p.batch * p.n_kv_heads + head) * p.capacity + j] = sum;
    else if (!p.accumulate)
      weights[j] = live[kb] ? sum : 0.f;
    else if (live[kb])
      weights[j] += sum;
  }
}

// Sum of the workgroups' shares of the rows, a slot per thread.  Slots from the length on
// have none; a key in a block outside the pool has no weight, whatever was taken for it.
template <bool kPaged>
__global__ __launch_bounds__(kThreads) void sum_kernel(const AttendParams p, const Divisor by_blocks, const uint32_t blocks) {
  const uint32_t head = by_blocks.divide(blockIdx.x);
  const int b = static_cast<int>(p.by_heads.divide(head));
  const int j = static_cast<int>(blockIdx.x - head * blocks) * kThreads + static_cast<int>(threadIdx.x);
  if (j >= p.capacity) return;
  const int64_t at = static_cast<int64_t>(head) * p.capacity + j;
  if (j >= clamp_length(p.cache_len[b], p.capacity)) {
    if (!p.accumulate) p.weights[at] = 0.f;
    return;
  }
  const int64_t step = static_cast<int64_t>(p.batch) * p.n_kv_heads * p.capacity;
  bool live = true;
  if constexpr (kPaged) {
    const int32_t blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + j / p.block_size];
    live = blk >= 0 && blk < p.n_blocks;
  }
  double sum = 0.0;
  for (int s = 0; s < p.n_split; ++s) sum += static_cast<double>(p.part[s * step + at]);
  const float w = live ? static_cast<float>(sum) : 0.f;
  p.weights[at] = p.accumulate ? p.weights[at] + w : w;
}

template <typename T, int D, bool kPaged, int kBlocks>
hipError_t weigh(const AttendParams &in, const WeightsPlan &plan, hipStream_t stream) {
  AttendParams p = in;
  p.n_slots = plan.n_stretches;
  p.n_split = plan.n_split;
  p.by_slot = Divisor::of(p.n_slots);
  p.by_split = Divisor::of(p.n_split);
  const int64_t heads = static_cast<int64_t>(p.n_kv_heads) * p.batch;
  const int64_t blocks = heads * p.n_slots * p.n_split, of_head = (p.capacity + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX || !grid_fits(blocks, kThreads) || (p.n_split > 1 && !grid_fits(heads * of_head, kThreads)))
    return hipErrorInvalidConfiguration;
  key_weights_kernel<T, D, kPaged, kBlocks><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  sum_kernel<kPaged><<<static_cast<unsigned>(heads * of_head), kThreads, 0, stream>>>(
      p, Divisor::of(static_cast<int32_t>(of_head)), static_cast<uint32_t>(of_head));
  return hipGetLastError();
}

template <typename T, bool kPaged>
hipError_t weigh_dim(const AttendParams &p, const WeightsPlan &plan, int head_dim, hipStream_t stream) {
  if constexpr (sizeof(T) == 2)
    if (plan.blocks == 2)
      return head_dim == 64 ? weigh<T, 64, kPaged, 2>(p, plan, stream) : weigh<T, 128, kPaged, 2>(p, plan, stream);
  return head_dim == 64 ? weigh<T, 64, kPaged, 1>(p, plan, stream) : weigh<T, 128, kPaged, 1>(p, plan, stream);
}

}  // namespace

WeightsPlan plan_key_weights(int64_t capacity, int32_t batch, int32_t total_q, int32_t n_q_heads, int32_t n_kv_heads,
                             int32_t head_dim, int32_t window, prcr_dtype dtype) {
  WeightsPlan plan{};
  int64_t tokens = (static_cast<int64_t>(total_q) + batch - 1) / batch;
  if (window > 0) tokens = std::min<int64_t>(tokens, window);
  const int64_t rows = tokens * (n_q_heads / n_kv_heads);     // of a sequence and KV head, on average
  // Two key blocks a wave use a row tile's read for both, but make half as many workgroups: for
  // long runs, counted as rows times stretches of 128 keys.  bf16, 8 KV heads of 4 query heads:
  // 4 prompts of 2,560 tokens (6.6 million) take 185 us with two and 194 with one; one
  // prompt of 1,000 (0.3 million) 31 and 27; 250 tokens over 1,400 slots of 16 sequences
  // (1.4 million) 83 and 88.  (float32, whose keys would take 256 registers, has one.)
  auto stretches = [&](int64_t blocks) { return (capacity + kWaves * 32 * blocks - 1) / (kWaves * 32 * blocks); };
  const int64_t heads = static_cast<int64_t>(batch) * n_kv_heads;
  plan.blocks = dtype == PRCR_BF16 && rows * stretches(1) * heads >= 1500000 ? 2 : 1;
  plan.n_stretches = static_cast<int32_t>(stretches(plan.blocks));
  // The rows are shared out over as many workgroups as run at a time, two on every compute unit, of at
  // least two tiles each (one prompt of 250 tokens: 14.4 us in 7 shares, 27 in one), and
  // those of long runs finer still, because stretches see different numbers of rows (4 prompts of
  // 2,560, 352 stretches: 185 us in 6 shares, 200 in 4, 218 in 3, 413 in one).  Stretches behind a
  // sequence's length are counted too, since the lengths are on the device: with a capacity of 8,192 slots
  // those prompts take 296 us (2 shares), with 32,768 446 (one).
  const int64_t have = plan.n_stretches * heads, tiles = rows / (dtype == PRCR_BF16 ? 64 : 32);
  plan.n_split = static_cast<int32_t>(std::max<int64_t>(
      {1, std::min<int64_t>(512 / have, tiles / 2), std::min<int64_t>((2048 + have - 1) / have, tiles / 8)}));
  const int64_t elem = dtype == PRCR_F32 ? 4 : 2;
  plan.rotated_bytes = (static_cast<size_t>(total_q) * n_q_heads * head_dim * elem + 255) / 256 * 256;
  plan.bytes = plan.rotated_bytes;
  // (Of several shares there are less than 4,096 workgroups, so partial sums of 4,096 x 256 keys at most.)
  if (plan.n_split > 1) plan.bytes += static_cast<size_t>(plan.n_split) * batch * n_kv_heads * capacity * 4;
  return plan;
}

hipError_t launch_key_weights(const AttendParams &p, const WeightsPlan &plan, prcr_dtype dtype, int head_dim, bool paged,
                              hipStream_t stream) {
  if (dtype == PRCR_F32)
    return paged ? weigh_dim<float, true>(p, plan, head_dim, stream) : weigh_dim<float, false>(p, plan, head_dim, stream);
  return paged ? weigh_dim<uint16_t, true>(p, plan, head_dim, stream)
               : weigh_dim<uint16_t, false>(p, plan, head_dim, stream);
}

}  // namespace prcr
