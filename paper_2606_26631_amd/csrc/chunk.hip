// Attention of several new tokens per sequence over the active cache: with row i of
// sequence b's n_b rows at slot p = cache_len[b] - n_b + i,
//   out = sum over slots j <= p of exp(s_j - lse) v_j,  s_j = scale q' . k_j,
//   lse = log sum over slots j <= p of exp(s_j),
// q' the rotated query.  A whole prompt is the case n_b = cache_len[b].
//
// A workgroup takes a tile of rows of one sequence and KV head, 32 rows a wave, or, of few
// rows, 32 for all its waves; the rows of a KV head are its tokens' query heads, token by
// token, so that a tile reads the cache once for all heads of the group.  Tiles of keys and
// values go through LDS, two of them, the next one's loads in flight while the present one is
// used: a tile of 64 keys is used by 128 rows, so that LDS is filled at a quarter of what it
// is read at, and two workgroups, of up to 256 registers a lane, fit a compute unit.  The wave forms the scores
// transposed, K (32 keys) x Q^T (32 rows): a lane then holds scores of one row only (that
// of its product column), the running maximum and sum of the softmax are one register
// each, and the weights are, in the registers where they arise, the operand of the value
// product V^T x P^T, whose contraction may take the keys in any order.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;

// 16 bytes per lane from memory to LDS: lane l's go to `to` + 16 l.
__device__ __forceinline__ void load_to_lds(const char *from, char *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// The sequence of the workgroup that comes `order`-th, and what the tile has to know of it.  The
// last tiles, which of a prompt see the most keys, come first.  Up to 64 sequences are one round of loads,
// a sequence per lane (every round costs about a microsecond before the first key), and
// their tiles are counted: tile slots are one behind the other, the workgroups without one at the end.
// Between the others, such workgroups left dies idle: 64 sequences of 32 rows, every second slot
// empty, took 137 us (float32, 1,160 slots), and 80 so (now, with the scores in four sums, 90).  Of more sequences, sequence b has the slots from
// floor(q_off[b] G / M) + b on, enough of them for its rows' tiles of M.
struct Sequence {
  int b, tile;                               // and the workgroup's tile of its rows (none: below 0)
  Rows rows;
  int32_t len;
};
template <int M>
__device__ __forceinline__ int32_t first_slot(const AttendParams &p, int b, int32_t off) {
  return static_cast<int32_t>(static_cast<uint32_t>(min(max(off, 0), p.total_q)) * static_cast<uint32_t>(p.group) / M) + b;
}
// Sum over the lanes up to each: within rows of 16, then the rows' last lanes onto the next ones.
__device__ __forceinline__ int running_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // from 1, 2, 4, 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row 0's sum to row 1, 2's to 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // the lower half's to the upper one
  return x;
}
template <int M>
__device__ __forceinline__ Sequence sequence_of(const AttendParams &p, int lane, int order) {
  int lo = 0, n = p.batch;                   // among sequences lo .. lo + n - 1
  int slot = p.n_slots - 1 - order;
  const bool counted = n <= kWave;
  while (n > kWave) {                        // the last that starts by `slot`
    const int step = (n + kWave - 1) / kWave;
    const int b = lo + lane * step;
    const bool ok = lane * step < n && first_slot<M>(p, b, p.q_off[b]) <= slot;
    const int k = max(__popcll(__ballot(ok)) - 1, 0) * step;
    lo += k;
    n = min(step, n - k);
  }
  const int b = lo + min(lane, n - 1);
  const Rows rows = rows_of(p, b);
  const int32_t len = clamp_length(p.cache_len[b], p.capacity);
  int tile, k;
  if (counted) {
    const int tiles = lane < n ? (rows.n * p.group + M - 1) / M : 0;
    const int end = running_sum(tiles);
    slot = __builtin_amdgcn_readlane(end, kWave - 1) - 1 - order;
    tile = slot - (end - tiles);
    const uint64_t mine = __ballot(tile >= 0 && tile < tiles);
    k = mine != 0 ? __ffsll(static_cast<unsigned long long>(mine)) - 1 : 0;
  } else {
    tile = slot - first_slot<M>(p, b, rows.start);
    k = max(__popcll(__ballot(lane < n && tile >= 0)) - 1, 0);
  }
  Sequence s;
  s.b = __builtin_amdgcn_readfirstlane(lo + k);
  s.tile = __builtin_amdgcn_readlane(tile, k);
  s.rows = Rows{__builtin_amdgcn_readlane(rows.start, k), __builtin_amdgcn_readlane(rows.n, k), false};
  s.len = __builtin_amdgcn_readlane(len, k);
  return s;
}

// What a tile of the cache's rows in LDS looks like.  A row's 16-byte chunks are permuted
// by the row's number, so that the lanes of one read fall on different banks: key rows, which
// are read 32 rows at a time at one chunk, over the whole row; value rows, which are read 4
// (bf16) neighbouring rows at a time at 4 chunks, by steps of 4 chunks.
template <typename T, int D>
struct TileOf {
  static constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kRowBytes = D * static_cast<int>(sizeof(T));
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kBytes = kKeys * kRowBytes;
  static constexpr int kRowsPerLoad = kWave / kChunks;
  static constexpr int kLoads = kKeys / kRowsPerLoad;    // wave loads of a tile
  __device__ static constexpr int key_swizzle(int row) { return row & (kChunks - 1); }
  __device__ static constexpr int value_swizzle(int row) {
    if constexpr (sizeof(T) == 4) return 0;
    return kChunks == 16 ? (row & 3) << 2 : (row >> 1 & 1) << 2;
  }
};

// kFew: one tile of 32 rows for all four waves, which share out its keys' tiles.
template <typename T, int D, bool kPaged, bool kFew>
__global__ __launch_bounds__(kThreads, kFew ? 1 : 2) void chunk_kernel(const AttendParams p) {
  using Tile = TileOf<T, D>;
  constexpr bool kHalf = sizeof(T) == 2;     // bf16
  constexpr int M = kFew ? 32 : 32 * kWaves;
  constexpr int KT = Tile::kKeys, kRowBytes = Tile::kRowBytes;
  constexpr int KB = KT / 32;                // key blocks of a tile
  constexpr uint64_t kAll = KT == 64 ? ~uint64_t{0} : (uint64_t{1} << (KT % 64)) - 1;
  constexpr int DT = D / 32;                 // feature blocks
  constexpr int kBy = kFew ? 1 : kWaves;     // waves that load a tile
  constexpr int kMine = Tile::kLoads / kBy;  // loads of each operand per wave and tile
  // Two tiles in turn, or (kFew) one of each wave.
  __shared__ __align__(1024) char s_kv[kFew ? kWaves : 2][2][Tile::kBytes];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane & 31, half = lane / 32;
  // The lane's rotary pair (one wave read of the arguments, in flight from the start).
  const double freq = p.inv_freq[lane % (D / 2)];
  const int axis = p.axis[lane % (D / 2)];
  if (blockIdx.x == 0 && p.err != nullptr) report(p, threadIdx.x, kThreads);
  const uint32_t id = blockIdx.x;
  const uint32_t by_head = p.by_heads.divide(id);
  const int kvh = static_cast<int>(id - by_head * static_cast<uint32_t>(p.n_kv_heads));
  const uint32_t by_split = p.by_split.divide(by_head);
  const int split = static_cast<int>(by_head - by_split * static_cast<uint32_t>(p.n_split));
  const Sequence seq = sequence_of<M>(p, lane, static_cast<int>(by_split));
  const int b = seq.b;
  const Rows rows = seq.rows;
  const int32_t len = seq.len;
  const int G = p.group;
  const int n_rows = rows.n * G;
  if (seq.tile < 0) return;
  const int r0 = seq.tile * M;
  if (r0 >= n_rows) return;

  const int first = len - rows.n;            // slot of the sequence's first row
  auto token_of = [&](int r) -> int { return static_cast<int>(p.by_group.divide(static_cast<uint32_t>(r))); };
  const int kend = first + token_of(min(r0 + M, n_rows) - 1) + 1;   // (at most len)
  const int n_tiles = max((kend + KT - 1) / KT, 0);
  const int per = (n_tiles + p.n_split - 1) / p.n_split;
  const int t0 = min(split * per, n_tiles), t1 = min(t0 + per, n_tiles);

  // The lane's row, and the last slots that it and the wave's last row see.
  const int wr0 = kFew ? r0 : r0 + wave * 32;
  const bool active = wr0 < n_rows;
  const int r = min(wr0 + l32, n_rows - 1);
  const int token = token_of(r);
  const int64_t row = (static_cast<int64_t>(rows.start) + token) * p.n_q_heads + kvh * G + (r - token * G);
  const int limit = first + token;
  const int wmax = __builtin_amdgcn_readlane(limit, 31);

  constexpr int kQ = Tile::kChunks / 2;      // 16-byte chunks of the lane's half of a row: 2 i + half
  u32x4 q[kQ];
  {
    const char *const at = static_cast<const char *>(p.q) + row * kRowBytes;
#pragma unroll
    for (int i = 0; i < kQ; ++i)
      if (!kFew || i % (kQ / 2) % kWaves == wave) q[i] = load_nt(at + (2 * i + half) * 16);   // (kFew: those it turns)
  }
  // The rows' tokens, eight at a time, a wave's or (kFew) two of them; their positions on the
  // lane's axis (with 32 pairs, of every second one) are in flight before the tile is asked for.
  constexpr int P = D / 2, kShare = kWave / P;
  constexpr int kTokens = 8, kTurns = kTokens / kShare / (kFew ? kWaves : 1);
  static_assert(kTokens * P * 16 * kWaves <= 2 * Tile::kBytes && kTurns >= 1, "a wave's angles in its share of a tile's buffers");
  const int tok0 = __builtin_amdgcn_readfirstlane(token), tok1 = __builtin_amdgcn_readlane(token, 31);
  auto turned = [&](int i) -> int { return ((kFew ? wave * kTurns : 0) + i) * kShare + lane / P; };   // token of eight
  int32_t pos[kTurns];
  auto load_pos = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      pos[i] = p.q_pos[(static_cast<int64_t>(rows.start) + min(c0 + turned(i), tok1)) * 3 + axis];
  };
  load_pos(tok0);

  // Rows of a tile: every load is issued for a row that exists; rows past the sequence's last
  // one, or in a block outside the pool, are left out by the mask.
  const int64_t pool = static_cast<int64_t>(p.layer) * p.n_blocks * p.block_size;
  const int64_t base = (kPaged ? pool * p.n_kv_heads + kvh
                               : ((static_cast<int64_t>(b) * p.n_layers + p.layer) * p.n_kv_heads + kvh) * p.s_max) *
                       kRowBytes;
  const char *const base_k = static_cast<const char *>(p.cache_k) + base;
  const char *const base_v = static_cast<const char *>(p.cache_v) + base;
  const uint32_t row_step = kPaged ? static_cast<uint32_t>(p.n_kv_heads) * kRowBytes : kRowBytes;
  const int32_t *const table = kPaged ? p.block_table + static_cast<int64_t>(b) * p.max_blocks : nullptr;
  int bad_block = 0;
  // Slot in the layer's pool of key `lane % KT` of tile t; -1 in a block outside it.
  // (A pool's slots are at least 128 bytes each: below 2^32 of them.)
  auto entry_of = [&](int t, int32_t *off) -> int32_t {
    const int j = min(t * KT + lane % KT, len - 1);
    const int lb = p.block_shift >= 0 ? j >> p.block_shift : j / p.block_size;
    *off = j - lb * p.block_size;
    return table[lb];
  };
  int32_t entry = 0, entry_off = 0;
  const int in_load = lane / Tile::kChunks, chunk = lane % Tile::kChunks;
  auto load_tile = [&](int t, char (*to)[Tile::kBytes]) -> uint64_t {
    uint64_t live = ~uint64_t{0};
    uint32_t pool_slot = 0;
    if constexpr (kPaged) {
      const bool ok = entry >= 0 && entry < p.n_blocks;
      live = __ballot(ok);
      bad_block |= !ok && t * KT + lane % KT < len;
      pool_slot = ok ? static_cast<uint32_t>(entry) * static_cast<uint32_t>(p.block_size) +
                           static_cast<uint32_t>(entry_off) : 0u;
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int load = kFew ? i : i * kWaves + wave;
      const int at = load * Tile::kRowsPerLoad + in_load;        // the lane's row of the tile
      int64_t from;
      if constexpr (kPaged)
        from = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(pool_slot), at))) *
                                    row_step);
      else
        from = static_cast<int64_t>(min(t * KT + at, len - 1)) * row_step;
      load_to_lds(base_k + from + (chunk ^ Tile::key_swizzle(at)) * 16, to[0] + load * 1024);
      load_to_lds(base_v + from + (chunk ^ Tile::value_swizzle(at)) * 16, to[1] + load * 1024);
    }
    return live;
  };

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -FLT_MAX, l = 0.f;               // running maximum (base 2), the lane's own keys' sum

  // The wave's first tile, and the tiles from one of its own to the next.
  const int tw = kFew ? t0 + wave : t0;
  constexpr int kStep = kFew ? kWaves : 1;
  uint64_t live = ~uint64_t{0}, live_next = ~uint64_t{0};
  if (tw < t1) {
    if constexpr (kPaged) entry = entry_of(tw, &entry_off);
    live_next = load_tile(tw, s_kv[kFew ? wave : tw & 1]);
    if constexpr (kPaged) entry = entry_of(min(tw + kStep, t1 - 1), &entry_off);
  }

  // The rows are turned while the first tile comes: in double precision, rounded once to the
  // stored type, as prefill capture rotates the keys.  (The matrix products take operands
  // of that type, so a query is rounded to it at some point; rounded here, the scores are those
  // of two rows of the same kind, and their sums stay in float32.)  The tokens' cosines and
  // sines go through LDS (the second tile's buffer, a share of it for each wave), since the
  // rows of a group share them; a pair's place is permuted by the token, for the banks.  kFew:
  // the waves share that work too, and the turned rows pass through LDS to all of them.
  if (active && t0 < t1) {
    constexpr int kPer = Store<T>::kPerChunk;
    // A pair's cosine and sine, 16 bytes: doubles, or (bf16) as two floats each.
    typedef double f64x2 __attribute__((ext_vector_type(2)));
    __shared__ __align__(16) f64x2 s_angles[kFew ? kTokens * P : 1];
    __shared__ __align__(16) char s_turned[kFew ? 32 : 1][kRowBytes];
    f64x2 *const table = kFew ? s_angles
                              : reinterpret_cast<f64x2 *>(&s_kv[(t0 + 1) & 1][0][0] + wave * (2 * Tile::kBytes / kWaves));
    // The angles' writes before their reads, and those before the next ones' writes.
    auto sync = [&] {
      if constexpr (kFew)
        __syncthreads();
      else
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the wave's own)
    };
    for (int c0 = tok0; c0 <= tok1; c0 += kTokens) {
      const int n = min(kTokens, tok1 + 1 - c0);
      if (c0 != tok0) load_pos(c0);
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int tok = turned(i);
        if ((tok & -kShare) >= n) break;     // (past the last token: not read)
        double sn, cs;
        turn(static_cast<double>(pos[i]) * freq, &sn, &cs);
        if (p.negate) {
          cs = -cs;
          sn = -sn;
        }
        f64x2 both = {cs, sn};
        if constexpr (kHalf) both = __builtin_bit_cast(f64x2, split_angle(cs, sn));
        table[tok * P + (lane % P ^ (tok & 7))] = both;
      }
      sync();
      const int tok = token - c0;
      if (tok >= 0 && tok < n) {
#pragma unroll
        for (int i = 0; i < kQ / 2; ++i) {
          if (kFew && i % kWaves != wave) continue;
          f64x2 angle[kPer];
#pragma unroll
          for (int e = 0; e < kPer; ++e) angle[e] = table[tok * P + (((2 * i + half) * kPer + e) ^ (tok & 7))];
          if constexpr (kHalf) {
            f32x4 split[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) split[e] = __builtin_bit_cast(f32x4, angle[e]);
            turn_bf16(q[i], q[i + kQ / 2], split);
          } else {
            double cs[kPer], sn[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
              cs[e] = angle[e][0];
              sn[e] = angle[e][1];
            }
            u32x4 lo, hi;
            Store<T>::rotate(q[i], q[i + kQ / 2], cs, sn, lo, hi);
            q[i] = lo;
            q[i + kQ / 2] = hi;
          }
        }
      }
      sync();
    }
    if constexpr (kFew) {
      const int sw = Tile::key_swizzle(l32);
#pragma unroll
      for (int i = 0; i < kQ; ++i)
        if (i % (kQ / 2) % kWaves == wave) *reinterpret_cast<u32x4 *>(&s_turned[l32][((2 * i + half) ^ sw) * 16]) = q[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kQ; ++i) q[i] = *reinterpret_cast<const u32x4 *>(&s_turned[l32][((2 * i + half) ^ sw) * 16]);
    }
  }
  // One tile.  The first tiles, which every row sees whole, have neither the mask nor, between
  // their reads and products, what is done for it: kMasked is right for every tile.
  auto step = [&](int t, auto is_masked) {
    constexpr bool kMasked = decltype(is_masked)::value;
    // The tile's loads have arrived, in every wave (kFew: the wave's own), and every wave is done
    // with the other buffer.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (!kFew) __syncthreads();
    live = live_next;
    if (!kFew && t + 1 < t1) {
      live_next = load_tile(t + 1, s_kv[(t + 1) & 1]);
      if constexpr (kPaged) entry = entry_of(min(t + 2, t1 - 1), &entry_off);
    }
    const int k0 = t * KT;
    if (!active || (kMasked && k0 > wmax)) return;
    const char *const kt = s_kv[kFew ? wave : t & 1][0];
    const char *const vt = s_kv[kFew ? wave : t & 1][1];

    // Scores: lane's keys 32 kb + 8 (i / 4) + 4 half + i % 4 of row l32.
    f32x16 s[KB];
    [[maybe_unused]] f32x16 lost;              // float32, kFew: of the scores, in their addition
    const char *const krow = kt + l32 * kRowBytes;
    const int sw = Tile::key_swizzle(l32);     // (32 rows on, the same)
    if constexpr (kHalf) {
      // All of the tile's key operands are on their way before the first product waits for one.
      u32x4 k[KB][kQ];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < kQ; ++i)
          k[kb][i] = *reinterpret_cast<const u32x4 *>(krow + 32 * kb * kRowBytes + ((2 * i + half) ^ sw) * 16);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int i = 0; i < kQ; ++i)
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[kb][i]),
                                                          __builtin_bit_cast(bf16x8, q[i]), s[kb], 0, 0, 0);
      }
    } else {
      // In four sums: one sum of D products in a row is off by a unit in the last place of the
      // score (root mean square), which at scores of 30 and more is 1e-6 of a weight; these, added
      // up, by 0.4 of that (for 4 % of a call's time).  kFew, whose calls of one token have no
      // other rows to average over, keeps the additions' errors too: by a quarter (300 slots: 15.7
      // us instead of 13.5; without kFew the registers would not hold them).  The next sum's key
      // operands are on their way while one is formed, but for paged rows of 128 in quantity: there the
      // registers they take would spill (4 prompts of 1,500 tokens, 8 heads of 4: 692 us without, 693
      // with them; 400 tokens each on some 1,500 cached ones, blocks of 5: 445 and 448).
      constexpr int kGroup = kQ / 4;
      constexpr bool kAhead = D == 64 || !kPaged || kFew;
      u32x4 k[2][kGroup];
      auto read = [&](int g) {
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
          k[g % 2][i] = *reinterpret_cast<const u32x4 *>(krow + ((2 * (g * kGroup + i) + half) ^ sw) * 16);
      };
      read(0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (!kAhead && g > 0) read(g);
        if (kAhead && g + 1 < 4) read(g + 1);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
          const f32x4 a = __builtin_bit_cast(f32x4, k[g % 2][i]), x = __builtin_bit_cast(f32x4, q[g * kGroup + i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], x[e], sum, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float a = g == 0 ? 0.f : s[0][i], t = a + sum[i], b = t - a;
          if constexpr (kFew) lost[i] = g == 0 ? 0.f : lost[i] + ((a - (t - b)) + (sum[i] - b));
          s[0][i] = t;
        }
      }
    }
    uint64_t sees = kAll;                  // bit: key of the tile that the lane's row sees
    uint32_t mine[2] = {~0u, ~0u};         // from the lane's first key on
    auto seen = [&](int kb, int i) -> bool { return mine[kb] >> (8 * (i / 4) + i % 4) & 1; };
    if constexpr (kMasked) {
      const int n = min(limit - k0 + 1, KT);
      sees = n >= KT ? kAll : n <= 0 ? 0 : (uint64_t{1} << n) - 1;
      sees &= live;
      mine[0] = static_cast<uint32_t>(sees) >> (4 * half);
      mine[1] = static_cast<uint32_t>(sees >> 32) >> (4 * half);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = seen(kb, i) ? s[kb][i] : -FLT_MAX;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    mx = half_max(mx) * p.scale2;
    // A maximum that rose by less than 2^8 is left where it is: weights up to 2^8 lose nothing
    // in float32 sums or in bf16, and the sums need no factor.
    if (__any(mx > m + 8.f)) {
      const float mn = fmaxf(m, mx);
      const float corr = exp2_hw(m - mn);
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= corr;
      m = mn;
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = fmaf(s[kb][i], p.scale2, -m);
        if constexpr (!kHalf && kFew) x = fmaf(lost[i] == lost[i] ? lost[i] : 0.f, p.scale2, x);   // (scores that are infinite lose NaN)
        s[kb][i] = exp2_hw(x);
        if constexpr (kMasked) s[kb][i] = seen(kb, i) ? s[kb][i] : 0.f;
        l += s[kb][i];
      }

    // Values.  A key without weight must not reach the sums through a value that is not
    // finite (zero times it would be NaN): in a tile of which some row does not see
    // everything such values are taken as zero here, and added to the rows that see them.
    bool odd = false;
    if constexpr (kHalf) {
      // A lane's weights of 16 keys (step c) are keys 16 c + 4 half + 0..3 and 8 further on; the
      // transposing read gives it feature l32's values of the same ones.  The products take bf16: a
      // weight is rounded to it here, after it has gone into the sum.  Outputs are then off by 2.1 to 2.3
      // thousandths of their norm, of which rounding them alone makes 1.6; the rest would take a second
      // part of the weights, and half as many products again.
      u32x4 w[2 * KB];
#pragma unroll
      for (int c = 0; c < 2 * KB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[c][e] = pack_bf16(s[c / 2][8 * (c % 2) + 2 * e], s[c / 2][8 * (c % 2) + 2 * e + 1]);
      __builtin_amdgcn_sched_barrier(0);
      const int x = lane % 16 / 4;
      const char *const vrow = vt + (4 * half + x) * kRowBytes + (lane / 16 % 2 * 2 + lane % 4 / 2) * 16 + lane % 2 * 8;
      // Feature block d's operands: one block's reads are in flight while the last one's
      // products run (the compiler left to itself reads all of them first, and spills).
      auto read = [&](int d, u32x4 (&v)[2 * KB]) {
        const char *const at = vrow + ((4 * d) ^ Tile::value_swizzle(x)) * 16;
#pragma unroll
        for (int c = 0; c < 2 * KB; ++c)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            const u32x2 two = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(at + (16 * c + 8 * u) * kRowBytes)));
            v[c][2 * u] = two[0];
            v[c][2 * u + 1] = two[1];
          }
      };
      u32x4 v[2][2 * KB];
      read(0, v[0]);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if (d + 1 < DT) read(d + 1, v[(d + 1) % 2]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 2 * KB; ++c) {
          u32x4 &a = v[d % 2][c];
          if constexpr (kMasked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool lo = (a[e] & 0x7F80u) == 0x7F80u, hi = (a[e] & 0x7F800000u) == 0x7F800000u;
              odd |= lo | hi;
              a[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
            }
          }
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                         __builtin_bit_cast(bf16x8, w[c]), o[d], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float *const vrow =
            reinterpret_cast<const float *>(vt + (8 * (i / 4) + i % 4 + 4 * half) * kRowBytes);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          float v = vrow[32 * d + l32];
          if constexpr (kMasked) {
            const bool bad = (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u;
            odd |= bad;
            v = bad ? 0.f : v;
          }
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[0][i], o[d], 0, 0, 0);
        }
      }
    }
    if (kMasked && __any(odd)) {
      for (int j = 0; j < KT; ++j) {
        const bool in = sees >> j & 1;
        const char *const vrow = vt + j * kRowBytes;
        const int sw = Tile::value_swizzle(j);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int at = (32 * d + 8 * (i / 4) + 4 * half + i % 4) * static_cast<int>(sizeof(T));   // byte of the row
            const char *const from = vrow + ((at / 16) ^ sw) * 16 + at % 16;
            float v;
            if constexpr (kHalf)
              v = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(from)) << 16);
            else
              v = *reinterpret_cast<const float *>(from);
            const bool bad = (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u;
            o[d][i] += in && bad ? v : 0.f;
          }
      }
    }
  };
  // Tiles that the workgroup's first row sees whole.
  const int t_whole = min(t1, max(t0, (first + token_of(r0) + 1) / KT));
  // (kFew: the wave's next tile, once this one's buffer has been read.)
  auto next_tile = [&](int t) {
    if (!kFew || t + kStep >= t1) return;
    live_next = load_tile(t + kStep, s_kv[wave]);
    if constexpr (kPaged) entry = entry_of(min(t + 2 * kStep, t1 - 1), &entry_off);
  };
  int t = tw;
  for (; t < t_whole; t += kStep) {
    if (kPaged && (live_next & kAll) != kAll) break;         // (a block outside the pool; the same in every wave of a tile)
    step(t, std::false_type{});
    next_tile(t);
  }
  for (; t < t1; t += kStep) {
    step(t, std::true_type{});
    next_tile(t);
  }
  if (kPaged && p.err != nullptr && __any(bad_block) && lane == 0) atomicOr(p.err, PRCR_DERR_BLOCK);

  l = half_sum(l);
  if constexpr (kFew) {
    // The waves' sums, through the tiles' buffers; a thread then has 1 / 8 of a row's features.
    constexpr int kRow = D + 4, F = D / 8;   // floats (padded for the banks)
    __shared__ float s_m[kWaves][32], s_l[kWaves][32];
    static_assert(32 * kRow * 4 <= 2 * Tile::kBytes, "a wave's sums in its tile's buffers");
    float *const mine = reinterpret_cast<float *>(&s_kv[wave][0][0]);
    if (half == 0) {
      s_m[wave][l32] = m;
      s_l[wave][l32] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4 *>(mine + l32 * kRow + 32 * d + 8 * i + 4 * half) =
            f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    __syncthreads();
    const int at = threadIdx.x / 8, from = static_cast<int>(threadIdx.x) % 8 * F;
    if (r0 + at >= n_rows) return;
    float ms = -FLT_MAX, ls = 0.f, x[F] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) ms = s_l[w][at] != 0.f ? fmaxf(ms, s_m[w][at]) : ms;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float lw = s_l[w][at];
      if (lw == 0.f) continue;               // (no key: no features either)
      const float f = exp2_hw(s_m[w][at] - ms);
      ls = fmaf(lw, f, ls);
      const float *const o_w = reinterpret_cast<const float *>(&s_kv[w][0][0]) + at * kRow + from;
#pragma unroll
      for (int e = 0; e < F; ++e) x[e] = fmaf(o_w[e], f, x[e]);
    }
    const int tok = token_of(r0 + at);
    const int64_t of = (static_cast<int64_t>(rows.start) + tok) * p.n_q_heads + kvh * G + (r0 + at - tok * G);
    if (p.n_split > 1) {
      float *const part = p.part + (of * p.n_split + split) * (D + 2);
      if (from == 0) {
        part[D] = ms;
        part[D + 1] = ls;
      }
#pragma unroll
      for (int e = 0; e < F; e += 2) *reinterpret_cast<f32x2 *>(part + from + e) = f32x2{x[e], x[e + 1]};
      return;
    }
    if (p.lse != nullptr && from == 0)
      p.lse[of] = ls != 0.f ? (ms + __builtin_amdgcn_logf(ls)) * 0.693147180559945309f : -__builtin_inff();
    char *const out = static_cast<char *>(p.out) + of * kRowBytes + from * static_cast<int>(sizeof(T));
#pragma unroll
    for (int e = 0; e < F; ++e) x[e] = ls != 0.f ? x[e] / ls : 0.f;
    if constexpr (kHalf) {
#pragma unroll
      for (int e = 0; e < F; e += 4)
        *reinterpret_cast<u32x2 *>(out + 2 * e) = u32x2{pack_bf16(x[e], x[e + 1]), pack_bf16(x[e + 2], x[e + 3])};
    } else {
#pragma unroll
      for (int e = 0; e < F; e += 4) *reinterpret_cast<f32x4 *>(out + 4 * e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
    }
    return;
  }
  if (!active || wr0 + l32 >= n_rows) return;
  if (p.n_split > 1) {
    float *const part = p.part + (row * p.n_split + split) * (D + 2);
    if (half == 0) {
      part[D] = m;
      part[D + 1] = t0 < t1 ? l : 0.f;
    }
    if (t0 >= t1) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 32 * d + 8 * i + 4 * half;
        *reinterpret_cast<f32x2 *>(part + at) = f32x2{o[d][4 * i], o[d][4 * i + 1]};
        *reinterpret_cast<f32x2 *>(part + at + 2) = f32x2{o[d][4 * i + 2], o[d][4 * i + 3]};
      }
    return;
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;   // (a NaN stays one)
  if (p.lse != nullptr && half == 0)
    p.lse[row] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.693147180559945309f : -__builtin_inff();
  char *const out = static_cast<char *>(p.out) + row * kRowBytes;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = l != 0.f ? o[d][4 * i + e] * inv : 0.f;
      const int at = 32 * d + 8 * i + 4 * half;
      if constexpr (kHalf)
        *reinterpret_cast<u32x2 *>(out + at * 2) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      else
        *reinterpret_cast<f32x4 *>(out + at * 4) = x;
    }
}

// Merge of a row's partial results: a wave per row, D / 64 features a lane.  The splits'
// maxima and sums are read a split per lane, and the features of kPre splits at once with them:
// one round of loads where there are no more.  Splits without keys have a sum of zero, and no
// features.
constexpr int kMergeWaves = 4;
constexpr int kMostSplits = kWave;
constexpr int kPre = 8;
template <typename T, int D>
__global__ __launch_bounds__(kMergeWaves * kWave) void merge_kernel(const AttendParams p) {
  constexpr int F = D / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kMergeWaves + threadIdx.x / kWave;
  if (row >= static_cast<int64_t>(p.total_q) * p.n_q_heads) return;
  const float *const part = p.part + row * p.n_split * (D + 2);
  auto at = [&](int s) -> const float * { return part + min(s, p.n_split - 1) * (D + 2); };
  const float m = at(lane)[D], l = lane < p.n_split ? at(lane)[D + 1] : 0.f;
  float o[kPre][F];
#pragma unroll
  for (int k = 0; k < kPre; ++k)
#pragma unroll
    for (int f = 0; f < F; ++f) o[k][f] = at(k)[f * kWave + lane];
  // Rows of no sequence have no partial results: the token lies behind its sequence's last row.
  const int32_t token = static_cast<int32_t>(p.by_row.divide(static_cast<uint32_t>(row)));
  int lo = 0, n = p.batch;                   // the last sequence that starts at or before the token
  bool mine = false;
  while (n > kWave) {
    const int step = (n + kWave - 1) / kWave;
    const int b = lo + lane * step;
    const bool ok = lane * step < n && p.q_off[b] <= token;
    const int k = max(__popcll(__ballot(ok)) - 1, 0) * step;
    lo += k;
    n = min(step, n - k);
  }
  if (lane < n) {
    const Rows rows = rows_of(p, lo + lane);
    mine = token >= rows.start && token < rows.start + rows.n;
  }
  if (!__any(mine)) return;
  const float M = wave_max(l != 0.f ? m : -FLT_MAX);
  const float w = l != 0.f ? exp2_hw(m - M) : 0.f;
  const float L = wave_sum(l * w);
  float O[F] = {};
  for (int k0 = 0; k0 < p.n_split; k0 += kPre) {
    if (k0 > 0) {
#pragma unroll
      for (int k = 0; k < kPre; ++k)
#pragma unroll
        for (int f = 0; f < F; ++f) o[k][f] = at(k0 + k)[f * kWave + lane];
    }
#pragma unroll
    for (int k = 0; k < kPre; ++k) {
      if (k0 + k >= p.n_split) break;
      const float lk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(l), k0 + k));
      const float wk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), k0 + k));
#pragma unroll
      for (int f = 0; f < F; ++f) O[f] = lk != 0.f ? fmaf(o[k][f], wk, O[f]) : O[f];
    }
  }
  if (lane == 0 && p.lse != nullptr)
    p.lse[row] = L != 0.f ? (M + __builtin_amdgcn_logf(L)) * 0.693147180559945309f : -__builtin_inff();
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const float x = L != 0.f ? O[f] / L : 0.f;
    if constexpr (sizeof(T) == 2)
      static_cast<uint16_t *>(p.out)[row * D + f * kWave + lane] = static_cast<uint16_t>(pack_bf16(x, 0.f));
    else
      static_cast<float *>(p.out)[row * D + f * kWave + lane] = x;
  }
}

template <typename T, int D, bool kPaged>
hipError_t chunk(const AttendParams &p, const ChunkPlan &plan, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(p.n_kv_heads) * p.n_slots * p.n_split;
  const int64_t rows = static_cast<int64_t>(p.total_q) * p.n_q_heads;
  const int64_t merges = (rows + kMergeWaves - 1) / kMergeWaves;
  if (blocks > INT32_MAX || !grid_fits(blocks, kThreads) || (p.n_split > 1 && !grid_fits(merges, kMergeWaves * kWave)))
    return hipErrorInvalidConfiguration;
  if (plan.few)
    chunk_kernel<T, D, kPaged, true><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  else
    chunk_kernel<T, D, kPaged, false><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  merge_kernel<T, D><<<static_cast<unsigned>(merges), kMergeWaves * kWave, 0, stream>>>(p);
  return hipGetLastError();
}

template <typename T, bool kPaged>
hipError_t chunk_dim(const AttendParams &p, const ChunkPlan &plan, int head_dim, hipStream_t stream) {
  return head_dim == 64 ? chunk<T, 64, kPaged>(p, plan, stream) : chunk<T, 128, kPaged>(p, plan, stream);
}

}  // namespace

ChunkPlan plan_chunk(int64_t capacity, int32_t batch, int32_t total_q, int32_t n_q_heads, int32_t n_kv_heads,
                     int32_t head_dim) {
  ChunkPlan plan{};
  const int64_t group = n_q_heads / n_kv_heads;
  const int64_t rows = static_cast<int64_t>(total_q) * group;
  // Workgroups for all rows and heads in tiles of m rows, of sequences of the same length.
  auto tiles = [&](int64_t m) { return std::max<int64_t>(batch * ((rows + m * batch - 1) / (m * batch)) * n_kv_heads, 1); };
  // Tiles of 32 rows whose keys the waves share out take a compute unit each (their LDS): where
  // one round of them does it.  bf16, 8 KV heads of 4 query heads, 4,000 cached slots, both ways:
  // one sequence of 40 rows, 40 workgroups, 18 and 21 us; 16 sequences of 16, 256 workgroups, 52
  // and 58; 4 sequences of 120, 480 workgroups, 73 and 59.
  plan.few = tiles(32) <= 256;
  const int64_t tile = plan.few ? 32 : 32 * kWaves, have = tiles(tile);
  plan.n_slots = static_cast<int32_t>(rows / tile) + batch;
  // The keys are split for as many workgroups as run at a time (few rows: one per
  // compute unit, else two), or, of fewer, by what that costs: a workgroup takes about a
  // microsecond for 64 keys (of each wave, where they share them out), and every split
  // writes and reads a partial result of 4 (D + 2) bytes per row and head, at some 16 MB a
  // microsecond, or 4 MB where a workgroup writes those of 128 rows at its end (of bf16 and the heads
  // above, one sequence of 40 rows over 1,192 slots: 13.0 us in 5 splits, 16.3 in 2; of 400 rows over
  // 500 slots: 21 us in one, 26 in 4; over 1,552 slots: 39 in one, 33 in 2, 34 in 4, 73 in 16).  The merge is
  // a launch more, about four microseconds: two rounds or fewer are not split.  A round that is
  // not full is better than two: one sequence of 400 rows over 4,400 slots, 104 workgroups, takes
  // 55 us in 4 splits, 66 in 5.  (The lengths are on the device: the capacity stands for them.  Float32,
  // whose tiles are of 32 keys and take longer, goes by the same rule, which was not measured for it.)
  const int64_t keys = plan.few ? 64 * kWaves : 64;          // of a workgroup at a time
  const double rounds = static_cast<double>(capacity) / keys, rows_all = static_cast<double>(total_q) * n_q_heads;
  const double best = rounds <= 2 ? 1 : std::sqrt(rounds * (plan.few ? 16e6 : 4e6) / (rows_all * 8 * (head_dim + 2)));
  const int64_t most = std::min<int64_t>({(plan.few ? 256 : 512) / have, (capacity + keys - 1) / keys, kMostSplits});
  plan.n_split = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(most, static_cast<int64_t>(best))));
  // (Of several splits there are at most 512 workgroups, so partial results of at most 512 x 128 rows.)
  if (plan.n_split > 1) plan.bytes = static_cast<size_t>(total_q) * n_q_heads * plan.n_split * (head_dim + 2) * 4;
  return plan;
}

hipError_t launch_chunk(const AttendParams &in, const ChunkPlan &plan, prcr_dtype dtype, int head_dim, bool paged,
                        hipStream_t stream) {
  AttendParams p = in;
  p.n_slots = plan.n_slots;
  p.n_split = plan.n_split;
  p.by_split = Divisor::of(plan.n_split);
  p.by_row = Divisor::of(p.n_q_heads);
  if (dtype == PRCR_F32)
    return paged ? chunk_dim<float, true>(p, plan, head_dim, stream) : chunk_dim<float, false>(p, plan, head_dim, stream);
  return paged ? chunk_dim<uint16_t, true>(p, plan, head_dim, stream)
               : chunk_dim<uint16_t, false>(p, plan, head_dim, stream);
}

}  // namespace prcr
