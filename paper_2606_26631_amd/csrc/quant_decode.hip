// Decode attention over the decoder cache in 8 bits (Eq. (14), as decode.hip has it): for each
// sequence and query head, with q' the query turned at its position times scale log2(e), in float32,
//   s_j = kscale_j (q' . kcode_j),   out = sum_j 2^(s_j - m) vscale_j vcode_j / sum_j 2^(s_j - m)
// over the slots below the sequence's length.  Split-K as there: one workgroup per key chunk, KV
// head and sequence, and the same merge of the chunks' partials.
//
// Both contractions run on the matrix cores, 32 keys at a time, as decode_partial_bf16_kernel's:
// a code (e4m3: 4 significant bits, int8: 7) is exactly a bf16 number, and the float32 operands
// are split into three bf16 parts whose sum they are, so that the products are exact and their
// sums float32.  The key's scale multiplies the score, and the value's the weight before it is
// split: neither costs an operation per element.
//
// What bounds it is reading the cache: 32 sequences of 2,756-4,256 keys, 8 heads, 237 MB, take 38 us at
// 6.2 TB/s and 4.7 in the merge, 64 paged ones of 2,912-6,512 in int8, 4 heads, 319 MB, 58.9 (5.4 TB/s) and
// 4.8.  Eight codes a lane on the vector ALU, with the scores summed across lanes, took 115 and 383.
// int8 keys multiplied as integers, with the query in four digits, were no faster (61.8 and 61.7 us a call).
#include <algorithm>
#include <type_traits>

#include "attend.h"
#include "decode_split.h"
#include "quant.h"

namespace prcr {
namespace {

// Two codes of a word (its lower or upper half) as two bf16 numbers.
template <bool kE4M3, bool kUpper>
__device__ __forceinline__ uint32_t codes2(uint32_t w) {
  if constexpr (kE4M3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, kUpper));
  } else {
    const float a = static_cast<float>(static_cast<int8_t>(w >> (kUpper ? 16 : 0)));
    const float b = static_cast<float>(static_cast<int8_t>(w >> (kUpper ? 24 : 8)));
    return pack_hi(__float_as_uint(a), __float_as_uint(b));
  }
}

// GT: query heads per KV head there is room for (4 or 8; smaller groups repeat their first head).
// kHalfBlocks (paged only): block_size is a multiple of 16, so that each half of a tile (tiles
// start at multiples of 32) lies in one block; other block sizes look every key up.
// kHeads: KV heads of a workgroup, whose waves are shared out to them (plan).
template <int D, int GT, bool kPaged, bool kHalfBlocks, bool kE4M3, int kWaves, int kHeads>
__global__ __launch_bounds__(kWaves * kWave, 2) void quant_decode_kernel(const QuantDecodeParams p) {
  constexpr int KK = D / 32;                 // products over the head dim per 16 keys
  constexpr int kKL = D / 64;                // key loads of 16 bytes per lane and 16 keys
  constexpr int kA = GT / 4;                 // query operands: 4 heads x (3 parts + 1 unused row)
  constexpr int kPT = GT / 4;                // weight operands of 16 rows
  constexpr int kPRows = 3 * GT + (GT == 4 ? 4 : 0);   // weight rows in LDS
  constexpr int kDL = D / 16;                // value features per lane
  constexpr int kVW = kDL / 4;               // words of their codes
  constexpr int kVL = kTile / 4;             // value loads per lane and tile (4 rows each)
  constexpr int kOwn = kWaves / kHeads;      // waves of a head
  constexpr int KPB = kOwn * kTile;          // keys per round of tiles
  constexpr int P = D / 2;
  constexpr int kQ = (GT * P + kOwn * kWave - 1) / (kOwn * kWave);   // query pairs per thread
  constexpr int kPS = kTile / 2 + 4;         // words per weight row in LDS, padded (decode.hip)
  typedef uint32_t vrow __attribute__((ext_vector_type(kVW)));
  __shared__ __align__(16) uint16_t s_q[kHeads][3 * GT][D + 8];
  __shared__ __align__(16) uint32_t s_p[kWaves][kPRows][kPS];
  __shared__ float s_m[kWaves][GT];
  __shared__ float s_l[kWaves][GT];
  __shared__ __align__(16) float s_o[kWaves][16][D];

  // Paged rows of 64 codes: two heads of a slot share a cache line.  Their workgroups are 8 apart, on one
  // chip die (workgroups are dealt to the 8 dies in turn), and read through its cache, so that the line comes
  // from memory once: 64 sequences of 2,000-4,000 keys, 8 heads of 64, 74 us, and 56 so (61 with reads past
  // the caches, 71 without the order).
  constexpr bool kHalfLines = D == 64 && kPaged;
  int kvh = blockIdx.x, row_y = blockIdx.y;
  if constexpr (kHalfLines && kHeads == 1) {
    const uint32_t id = blockIdx.x + gridDim.x * blockIdx.y, heads = gridDim.x;
    if (heads % 2 == 0 && id < heads * gridDim.y / 16 * 16) {
      const uint32_t pair = id / 16 * 8 + id % 8;
      kvh = static_cast<int>(2 * (pair % (heads / 2)) + id / 8 % 2);
      row_y = static_cast<int>(pair / (heads / 2));
    }
  }
  const int split = blockIdx.z;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int head = wave / kOwn, thread = threadIdx.x - head * kOwn * kWave;   // of the workgroup's heads, and in its waves
  kvh = kvh * kHeads + head;
  const double inv = p.inv_freq[thread % P];
  int len_in;
  const int b = sequence_of_row<kWaves>(p, lane, row_of(p, split, row_y), &len_in);
  const int n16 = lane % 16;                 // product column; operand row
  const int kj = lane / 16;                  // k group of the operands; head of the lane's scores
  const int G = p.group;

  const int len = clamp_len(p, kPaged, len_in);
  if (len != len_in && split == 0 && kvh == 0 && thread == 0 && p.err != nullptr)
    atomicOr(p.err, PRCR_DERR_CAPACITY);
  const int chunk = chunk_keys(p, len);
  const int j0 = static_cast<int>(min(static_cast<int64_t>(len), static_cast<int64_t>(split) * chunk));
  const int j1 = static_cast<int>(min(static_cast<int64_t>(len), static_cast<int64_t>(j0) + chunk));
  if (j0 >= j1 && split > 0) return;

  // The query's rows, before the first tile's: their wait does not wait for those.
  const int32_t q_pos = p.q_pos[b];
  float q_lo[kQ], q_hi[kQ];
#pragma unroll
  for (int u = 0; u < kQ; ++u) {
    const int g = u * (kOwn * kWave / P) + thread / P;
    const int64_t row = (static_cast<int64_t>(b) * p.n_q_heads + kvh * G + (g < G ? g : 0)) * D + thread % P;
    if (p.q_f32) {
      q_lo[u] = static_cast<const float *>(p.q)[row];
      q_hi[u] = static_cast<const float *>(p.q)[row + P];
    } else {
      q_lo[u] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(p.q)[row]) << 16);
      q_hi[u] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(p.q)[row + P]) << 16);
    }
  }

  // Keys of a tile.  Column n16 of score product st is key 8 (n16/4) + 4 st + n16%4, value load
  // u holds key 4 u + kj: both put key t at position (t % 4) * 8 + t / 4 of the value product's
  // contraction, with a lane's two scores in one word.  Lane l looks after one key of the tile,
  // that of its column and st = kj % 2: its table entry, whether it counts, and a scale.
  const int mine = 8 * (n16 / 4) + 4 * (kj % 2) + n16 % 4;
  auto lane_of = [](int t) -> int { return 16 * (t / 4 % 2) + 4 * (t / 8) + t % 4; };
  const int64_t row_layer = static_cast<int64_t>(p.layer) * p.n_blocks * p.block_size;   // paged
  const int64_t row_any = kPaged ? row_layer * p.n_kv_heads + kvh
                                 : ((static_cast<int64_t>(b) * p.n_layers + p.layer) * p.n_kv_heads + kvh) * p.s_max;
  const int64_t scale_any = kPaged ? (row_layer * p.n_kv_heads + static_cast<int64_t>(kvh) * p.block_size) : row_any;
  const char *const cache_k = static_cast<const char *>(p.cache_k);
  const char *const cache_v = static_cast<const char *>(p.cache_v);
  const float *const scales = kj < 2 ? p.k_scale : p.v_scale;
  int bad_block = 0;

  // Table entry of the lane's key of the tile at tb (the sequence's first entry past the chunk),
  // and the key's offset in its block.  Entries are read two tiles ahead, so that the loads that
  // need one never wait for it.
  struct Entry {
    int32_t blk, off;
  };
  auto entry_of = [&](int tb) -> Entry {
    Entry e{0, 0};
    if constexpr (kPaged) {
      const int j = tb + mine, js = j < j1 ? j : 0;
      const int lb = p.block_shift >= 0 ? (js >> p.block_shift) : js / p.block_size;
      e.blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + lb];
      e.off = js - lb * p.block_size;
    }
    return e;
  };
  // Rows of a tile.  Every load is issued unconditionally: keys past the chunk, or in a block
  // outside the pool, read a row that exists and are left out of `live` (bit l < 32: lane l's key).
  //   contiguous     one base; key t is row min(t, last)
  //   half blocks    one base per half; key t is row min(t % 16, last[t / 16])
  //   other blocks   lane l holds its key's slot in the layer's pool (below 2^32)
  struct TileRows {
    int64_t base[2];
    int last[2];
    uint32_t slot;
    uint32_t live;
    int64_t scale;                           // of the lane's key
  };
  auto rows_of = [&](int tb, Entry e) -> TileRows {
    TileRows t{};
    const bool in = mine < j1 - tb;
    if constexpr (!kPaged) {
      t.live = static_cast<uint32_t>(__ballot(in));
      const int tc = max(min(tb, j1 - 1), 0);
      t.base[0] = row_any + tc;
      t.last[0] = max(j1 - 1 - tc, 0);
      t.scale = t.base[0] + min(mine, t.last[0]);
    } else {
      const bool ok = in && e.blk >= 0 && e.blk < p.n_blocks;
      const uint32_t live = static_cast<uint32_t>(__ballot(ok));   // lanes l and l + 32 agree
      bad_block |= live != static_cast<uint32_t>(__ballot(in));
      t.live = live;
      const int64_t slot = static_cast<int64_t>(e.blk) * p.block_size + e.off;
      t.scale = ok ? scale_any + (slot - e.off) * p.n_kv_heads + e.off : scale_any;
      if constexpr (kHalfBlocks) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t lh = live & (h == 0 ? 0x00FF00FFu : 0xFF00FF00u);   // keys 16 h to 16 h + 15
          const int first = 8 * h;           // lane_of(16 h)
          const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(slot), first);
          const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(slot >> 32), first);
          const int64_t s = static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
          t.base[h] = lh != 0 ? (row_layer + s) * p.n_kv_heads + kvh : row_any;
          t.last[h] = lh != 0 ? __popc(lh) - 1 : 0;
        }
      } else {
        t.slot = ok ? static_cast<uint32_t>(slot) : 0u;
      }
    }
    return t;
  };
  const uint32_t row_step = kPaged ? static_cast<uint32_t>(p.n_kv_heads) * D : D;   // (below 2^23)
  // Where byte `at` of key t's row is in an array (t / 16 == half): a base that all lanes share, and
  // 32 bits of a lane's own.
  auto in_row = [&](const char *cache, const TileRows &tr, int t, int half, uint32_t at) -> const char * {
    if constexpr (!kPaged) {
      const char *const base = cache + tr.base[0] * D;
      return base + (static_cast<uint32_t>(min(t, tr.last[0])) * D + at);
    } else if constexpr (kHalfBlocks) {
      const char *const base = cache + tr.base[half] * D;
      return base + (__umul24(static_cast<uint32_t>(min(t - 16 * half, tr.last[half])), row_step) + at);
    } else {
      const uint32_t slot = static_cast<uint32_t>(__shfl(static_cast<int>(tr.slot), lane_of(t)));
      return cache + (row_layer + static_cast<int64_t>(slot)) * row_step + (static_cast<uint32_t>(kvh) * D + at);
    }
  };
  // Key rows, whole lines once, past the caches: load 0 of 128 features reads the rows of columns
  // 0..7, load 1 those of columns 8..15, a half of a row in the lanes of its own column and the
  // other 8 lanes away (swap_rows8 brings it over).  Of 64 features a load reads 16 whole rows.
  const int ka = 8 * (n16 % 8 / 4) + n16 % 4;
  auto load_k = [&](const TileRows &tr, u32x4 (&kd)[2][kKL]) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      if constexpr (kKL == 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          kd[st][u] = load_nt(in_row(cache_k, tr, ka + 4 * st + 16 * u, u, (n16 / 8) * 64 + kj * 16));
      } else {
        const int t = 8 * (n16 / 4) + 4 * st + n16 % 4;
        const char *const lo = in_row(cache_k, tr, t, 0, kj * 16), *const hi = in_row(cache_k, tr, t, 1, kj * 16);
        const char *const at = n16 < 8 ? lo : hi;
        kd[st][0] = kHalfLines ? *reinterpret_cast<const u32x4 *>(at) : load_nt(at);   // (one of them is the key's)
      }
    }
  };
  // Value rows, 16 lanes to a row.
  auto load_v = [&](const TileRows &tr, vrow (&vd)[kVL]) {
#pragma unroll
    for (int u = 0; u < kVL; ++u) {
      const vrow *const at = reinterpret_cast<const vrow *>(in_row(cache_v, tr, 4 * u + kj, u / 4, n16 * kDL));
      vd[u] = kHalfLines ? *at : __builtin_nontemporal_load(at);
    }
  };

  // The wave's tiles start at jw + n * KPB; the next tile's key rows are loaded once this tile's
  // products have read them, and its value rows once the value product has.
  const int jw = j0 + wave % kOwn * kTile;
  u32x4 kr[2][kKL];
  vrow vv[kVL];
  Entry e_next;
  TileRows tr;
  float sc_next;                             // the lane's key's scale: of its key row, or (kj >= 2) its value row
  {
    const Entry e0 = entry_of(jw);
    e_next = entry_of(jw + KPB);
    tr = rows_of(jw, e0);
    sc_next = scales[tr.scale];
    load_k(tr, kr);
    load_v(tr, vv);
  }

  // Turned, scaled query of every head of the group, in float32, as three bf16 parts in LDS.
  {
    const double qs = static_cast<double>(p.scale) * kLog2e;
    const int i = thread % P;
    double sn, cs;
    turn(static_cast<double>(q_pos) * inv, &sn, &cs);
#pragma unroll
    for (int u = 0; u < kQ; ++u) {
      const int g = u * (kOwn * kWave / P) + thread / P;
      if (g < GT) {
        const double x = q_lo[u], xp = q_hi[u];
        const float y = static_cast<float>((x * cs - xp * sn) * qs);
        const float yp = static_cast<float>((xp * cs + x * sn) * qs);
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          s_q[head][3 * g + part][i] = static_cast<uint16_t>(split_part(y, part) >> 16);
          s_q[head][3 * g + part][i + P] = static_cast<uint16_t>(split_part(yp, part) >> 16);
        }
      }
    }
  }
  lds_barrier();
  // Query operands: row n16 of operand a is part n16 % 4 of head 4 a + n16 / 4 (the fourth row
  // repeats the third; its scores are not used).  The lane's codes of a key are chunks kj and
  // kj + 4 of 16, its features of product kk the (kk % 2)-th half of chunk kj + 4 (kk / 2).
  u32x4 qa[kA][KK];
#pragma unroll
  for (int a = 0; a < kA; ++a) {
    const uint16_t *row = s_q[head][3 * (4 * a + n16 / 4) + min(n16 % 4, 2)];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qa[a][kk] = *reinterpret_cast<const u32x4 *>(row + 16 * (kj + 4 * (kk / 2)) + 8 * (kk % 2));
  }

  f32x4 acc[kDL];                            // rows 4 kj + r, features kDL * n16 + dt
#pragma unroll
  for (int dt = 0; dt < kDL; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mrun[kA], lsum[kA];                  // head 4 a + kj; lsum over the lane's own keys
#pragma unroll
  for (int a = 0; a < kA; ++a) {
    mrun[a] = -FLT_MAX;
    lsum[a] = 0.f;
  }

  for (int jt = jw; jt < j1; jt += KPB) {
    const uint32_t live = tr.live;
    f32x4 sa[kA][2];
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      if constexpr (kKL == 2) swap_rows8(kr[st][0], kr[st][kKL - 1]);
#pragma unroll
      for (int a = 0; a < kA; ++a) sa[a][st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint32_t w0 = kr[st][kk / 2][2 * (kk % 2)], w1 = kr[st][kk / 2][2 * (kk % 2) + 1];
        const u32x4 kb = {codes2<kE4M3, false>(w0), codes2<kE4M3, true>(w0), codes2<kE4M3, false>(w1),
                          codes2<kE4M3, true>(w1)};
#pragma unroll
        for (int a = 0; a < kA; ++a) sa[a][st] = mfma_16x16x32(qa[a][kk], kb, sa[a][st]);
      }
    }
    // The scales of the column's two keys: lanes' rows 0 and 1 hold the key rows', 2 and 3 the value rows'.
    float ks[2], vs[2];
    {
      const uint32_t x = __float_as_uint(sc_next);
      const auto half = __builtin_amdgcn_permlane32_swap(x, x, false, false);
      const auto k = __builtin_amdgcn_permlane16_swap(half[0], half[0], false, false);
      const auto v = __builtin_amdgcn_permlane16_swap(half[1], half[1], false, false);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        ks[st] = __uint_as_float(k[st]);
        vs[st] = __uint_as_float(v[st]);
      }
    }
    // (A tile past the chunk re-reads one row.)
    tr = rows_of(jt + KPB, e_next);
    e_next = entry_of(jt + 2 * KPB);
    sc_next = scales[tr.scale];
    load_k(tr, kr);

    const bool live0 = (live >> n16) & 1u, live1 = (live >> (16 + n16)) & 1u;
    vs[0] = live0 ? vs[0] : 0.f;
    vs[1] = live1 ? vs[1] : 0.f;
    float sc[kA][2];
    bool rise = false;
#pragma unroll
    for (int a = 0; a < kA; ++a) {
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const float s = ((sa[a][st][0] + sa[a][st][1]) + sa[a][st][2]) * ks[st];
        sc[a][st] = (st == 0 ? live0 : live1) ? s : -INFINITY;
        rise = rise || sc[a][st] > mrun[a];
      }
    }
    // The tile's maxima are needed only when some score rose above the running maximum of its
    // head (rarely, after the first tiles).
    if (__any(rise)) {
      float corr[kA];
#pragma unroll
      for (int a = 0; a < kA; ++a) {
        const float mnew = fmaxf(mrun[a], row_max16(fmaxf(sc[a][0], sc[a][1])));
        corr[a] = exp2_fast(mrun[a] - mnew);
        lsum[a] *= corr[a];
        mrun[a] = mnew;
      }
      // Accumulator row 4 kj + r belongs to head r (4 heads), or to head 4 (kj % 2) + r (8
      // heads); head h's factor is in lanes 16 (h % 4)...
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(corr[0]), 16 * r));
        if constexpr (kA == 2) {
          const float c1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(corr[kA - 1]), 16 * r));
          c = (kj & 1) ? c1 : c;
        }
#pragma unroll
        for (int dt = 0; dt < kDL; ++dt) acc[dt][r] *= c;
      }
    }
    // Weights, times the value rows' scales, as three bf16 parts, two keys to a word.
#pragma unroll
    for (int a = 0; a < kA; ++a) {
      uint32_t part[3][2];
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const float w = exp2_fast(sc[a][st] - mrun[a]);   // (0 where the key has no weight)
        lsum[a] += w;
#pragma unroll
        for (int q = 0; q < 3; ++q) part[q][st] = split_part(w * vs[st], q);
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const int row = GT == 4 ? 4 * q + kj : 8 * q + 4 * a + kj;
        s_p[wave][row][(n16 % 4) * 4 + n16 / 4] = pack_hi(part[q][0], part[q][1]);
      }
    }
    wave_lds_sync();
    u32x4 pa[kPT];
    pa[0] = *reinterpret_cast<const u32x4 *>(&s_p[wave][n16][4 * kj]);
    if constexpr (kPT == 2) {
      // (The second operand's other eight rows have no weight.)
      pa[kPT - 1] = *reinterpret_cast<const u32x4 *>(&s_p[wave][16 + n16 % 8][4 * kj]);
      const uint32_t keep = n16 < 8 ? ~0u : 0u;
#pragma unroll
      for (int w = 0; w < 4; ++w) pa[kPT - 1][w] &= keep;
    }
    // A zero weight times a code that is no number would make a NaN: codes of keys without weight are
    // taken as zero.
    if (live != ~0u) {
#pragma unroll
      for (int u = 0; u < kVL; ++u) {
        const uint32_t keep = (live >> lane_of(4 * u + kj)) & 1u ? ~0u : 0u;
#pragma unroll
        for (int w = 0; w < kVW; ++w) vv[u][w] &= keep;
      }
    }
    // Transposed value operand: feature kDL * n16 + dt of the lane's 8 keys, two keys' codes of
    // two features side by side and then turned into bf16.
#pragma unroll
    for (int f = 0; f < kVW; ++f) {
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        u32x4 vb[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t two = __builtin_amdgcn_perm(vv[2 * w + 1][f], vv[2 * w][f], pair == 0 ? 0x05010400u : 0x07030602u);
          vb[0][w] = codes2<kE4M3, false>(two);
          vb[1][w] = codes2<kE4M3, true>(two);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int q = 0; q < kPT; ++q)
            acc[4 * f + 2 * pair + e] = mfma_16x16x32(pa[q], vb[e], acc[4 * f + 2 * pair + e]);
      }
    }
    load_v(tr, vv);
  }
  if (bad_block && lane == 0 && p.err != nullptr) atomicOr(p.err, PRCR_DERR_BLOCK);

  // The lanes of a row of 16 hold different keys of one head.
#pragma unroll
  for (int a = 0; a < kA; ++a) {
    lsum[a] = group_sum<16>(lsum[a]);
    if (n16 == 0) {
      s_m[wave][4 * a + kj] = mrun[a];
      s_l[wave][4 * a + kj] = lsum[a];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
#pragma unroll
    for (int c = 0; c < kDL / 4; ++c)
      *reinterpret_cast<f32x4 *>(&s_o[wave][4 * kj + r][kDL * n16 + 4 * c]) =
          f32x4{acc[4 * c][r], acc[4 * c + 1][r], acc[4 * c + 2][r], acc[4 * c + 3][r]};
  }
  __syncthreads();
  finish_split<kOwn, D, GT, GT == 4 ? 3 : 2, GT>(p, b, kvh, G, split, thread,
                                                 *reinterpret_cast<const float(*)[kOwn][GT]>(&s_m[head * kOwn]),
                                                 *reinterpret_cast<const float(*)[kOwn][GT]>(&s_l[head * kOwn]),
                                                 *reinterpret_cast<const float(*)[kOwn][16][D]>(&s_o[head * kOwn]));
}

template <int D, int GT, bool kE4M3, int kWaves>
void launch_one(const QuantDecodeParams &p, bool paged, hipStream_t stream) {
  const dim3 grid(p.n_kv_heads / p.heads, p.batch, p.n_split), block(kWaves * kWave);
  const bool halves = paged && p.block_size % 16 == 0;
  if constexpr (D == 128 && kWaves == 4) {
    if (p.heads == 2) {
      if (halves)
        quant_decode_kernel<D, GT, true, true, kE4M3, kWaves, 2><<<grid, block, 0, stream>>>(p);
      else
        quant_decode_kernel<D, GT, true, false, kE4M3, kWaves, 2><<<grid, block, 0, stream>>>(p);
      return;
    }
  }
  if (!paged)
    quant_decode_kernel<D, GT, false, false, kE4M3, kWaves, 1><<<grid, block, 0, stream>>>(p);
  else if (halves)
    quant_decode_kernel<D, GT, true, true, kE4M3, kWaves, 1><<<grid, block, 0, stream>>>(p);
  else
    quant_decode_kernel<D, GT, true, false, kE4M3, kWaves, 1><<<grid, block, 0, stream>>>(p);
}

template <int D, int GT>
void launch_code(const QuantDecodeParams &p, prcr_code code, bool paged, hipStream_t stream) {
  if (code == PRCR_E4M3)
    p.waves == 8 ? launch_one<D, GT, true, 8>(p, paged, stream) : launch_one<D, GT, true, 4>(p, paged, stream);
  else
    p.waves == 8 ? launch_one<D, GT, false, 8>(p, paged, stream) : launch_one<D, GT, false, 4>(p, paged, stream);
}

// How a call is split, within the room for decode_splits' partials (p->n_split on entry).  As decode.hip's
// plan, only the sequence's length and the call's shape enter, and half the bytes a key move its borders:
//   - a cache of at most 1,024 slots (head_dim 64: 2,048) is one chunk a sequence: 8 sequences of 400-800
//     keys, 8 KV heads, take 9.4 us so, in chunks and a merge 10.4; one of 1,152 keys 10.2 and 9.9;
//   - else one workgroup per compute unit (head_dim 64: two; 8 sequences of 8,000 keys, 8 heads, 19.8 us with
//     eight chunks each, 23.3 with four), and two to four, of 1,024 keys and more, where there are several
//     sequences, which may differ in length: 64 of 2,912-6,512 keys, 4 KV heads, 62 us in two chunks and 69 in one
//     (32 of 2,756-4,256, 8 KV heads, 41 and 40; one of 120,001 42 in 32 and 43 in 64; 64 of
//     1,000-2,000, 4 KV heads, 25 in two and 23 in one).
// A sequence that is one chunk is read by eight waves where they are few, or have half the bytes a key
// (one of 600 keys: 7.7 us, with four waves 8.1; 32 of 1,000-2,000, 8 heads of 64: 11.7 and 14.3; but 64
// of 1,000-2,000, 4 heads of 128, 24.1 and 23.0).  More than about 42 GB/s a compute unit does not read.
//
// Paged rows of one head are 128 bytes here and there.  With 8 heads and more a workgroup takes two
// neighbouring ones, 256 bytes of a slot at about the same time: 16 sequences of 3,000-5,000 keys, 8
// heads, 31.3 us with one and 29.1 with two, 64 of 1,500-3,000 62.6 and 55.5 (contiguous: 25.0 with one,
// 25.8 with two; 64 of 2,912-6,512 keys, 4 heads, 62 either way; four heads are no better than two).
void plan(QuantDecodeParams *p, int head_dim, bool paged) {
  const int64_t capacity = paged ? static_cast<int64_t>(p->max_blocks) * p->block_size : p->s_max;
  const bool direct = capacity <= (head_dim == 64 ? 2048 : 1024);
  p->heads = !direct && paged && head_dim == 128 && p->n_kv_heads >= 8 && p->n_kv_heads % 2 == 0 ? 2 : 1;
  const int64_t room = p->n_split, pairs = static_cast<int64_t>(p->batch) * p->n_kv_heads / p->heads;
  constexpr int kMinKeys = 1024;
  int64_t fill = 1, n = 1;
  if (!direct) {
    const int64_t units = head_dim == 64 ? 2 * kUnits : kUnits;
    fill = pairs >= 3 * units / 4 ? 1 : splits_in_rounds(pairs, 3 * units / 4, 2 * units, room, 0.9);
    n = fill;
    if (p->batch > 1 && capacity / kMinKeys >= std::min(ceil_div(2 * kUnits, pairs), room)) {
      const int64_t more = splits_in_rounds(pairs, 2 * kUnits, 4 * kUnits, room, 0.9);
      if (capacity / kMinKeys >= more) n = std::max(fill, more);
    }
  }
  p->n_split = static_cast<int32_t>(n);
  p->fill = static_cast<int32_t>(fill);
  p->min_keys = kMinKeys / 2;                // (of a chunk of a shorter sequence)
  p->waves = n == 1 && p->heads == 1 && (head_dim == 64 || pairs <= kUnits / 2) ? 8 : 4;
  p->round = p->waves / p->heads * kTile;
  auto inverse = [](int64_t m) { return m > 1 ? static_cast<uint32_t>(((int64_t{1} << 32) + m - 1) / m) : 0u; };
  p->split_inverse = inverse(n);
  p->fill_inverse = inverse(fill);
  p->direct = n == 1;
}

}  // namespace

hipError_t launch_quant_decode(const QuantDecodeParams &in, prcr_code code, int head_dim, bool paged, hipStream_t stream) {
  QuantDecodeParams p = in;
  p.group = p.n_q_heads / p.n_kv_heads;
  plan(&p, head_dim, paged);
  if (head_dim == 64)
    p.group <= 4 ? launch_code<64, 4>(p, code, paged, stream) : launch_code<64, 8>(p, code, paged, stream);
  else
    p.group <= 4 ? launch_code<128, 4>(p, code, paged, stream) : launch_code<128, 8>(p, code, paged, stream);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.direct ? e : launch_decode_merge(p, head_dim, paged, stream);
}

}  // namespace prcr
