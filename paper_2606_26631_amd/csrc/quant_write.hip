// Writing the decoder cache in 8 bits: tokens' keys and values as a layer makes them (append),
// and revisited visual tokens from the memory in every layer (rebind).  A key row is turned at
// the token's position, as a cache of the rows' type holds it, and then it and the value row
// are quantised: their largest magnitude, the scale, the codes.
//
// A wave has its tokens side by side: 8 of 8 lanes each (bf16 rows of 128, float32 rows of 64), 16 of 4 (bf16, 64) or 4
// of 16 (float32, 128).  It goes through their rows (heads, or layers and heads), so that what it stores of a row
// are neighbouring slots: whole lines of codes, and scales next to each other.  A workgroup's waves share the tokens'
// angles (in double precision, in LDS) and take the rows in turn; keys and values are separate workgroups.  With a lane's
// angles computed by itself and keys and values in one wave, 8 prompts of 2,560 tokens took 29.3 us, now 25.0; 16 x
// 512 revisited tokens 158 and 143.  What bounds it is reading the rows and writing the codes (5.1 and 5.0 TB/s), of
// few tokens the dependent loads before a row: lengths, table entry and row in two rounds (64 paged tokens of
// 4 heads 4.7 us; a launch without a token 4.4).
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attend.h"
#include "quant.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kWaves = 4;

// Largest over the kLanes consecutive lanes that hold a row.
template <int kLanes>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  auto step = [&](auto ctrl) {
    return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, 0xF, 0xF, false)));
  };
  x = step(std::integral_constant<int, 0xB1>{});     // lane ^ 1
  x = step(std::integral_constant<int, 0x4E>{});     // lane ^ 2
  if constexpr (kLanes >= 8) x = step(std::integral_constant<int, 0x141>{});   // the other quad
  if constexpr (kLanes >= 16) x = step(std::integral_constant<int, 0x140>{});  // the other half
  return x;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef double f64x2 __attribute__((ext_vector_type(2)));

// Bits of the largest magnitude among a lane's elements of a row, E of each half, as float32.
template <typename T>
__device__ __forceinline__ uint32_t largest(u32x4 lo, u32x4 hi) {
  if constexpr (sizeof(T) == 2) {
    u16x2 most = {0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, static_cast<uint32_t>(lo[q] & 0x7FFF7FFFu)));
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, static_cast<uint32_t>(hi[q] & 0x7FFF7FFFu)));
    }
    return static_cast<uint32_t>(max(most[0], most[1])) << 16;
  } else {
    uint32_t most = 0u;
#pragma unroll
    for (int q = 0; q < 4; ++q) most = max(most, max(lo[q] & 0x7FFFFFFFu, hi[q] & 0x7FFFFFFFu));
    return most;
  }
}

// Four of a lane's elements of one half, from element 4 i on.
template <typename T>
__device__ __forceinline__ void elements(u32x4 w, int i, float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2)
      x[e] = __uint_as_float(e % 2 ? w[2 * i + e / 2] & 0xFFFF0000u : w[2 * i + e / 2] << 16);
    else
      x[e] = __uint_as_float(w[e]);
  }
}

// A row's scale, max(largest / Q, 2^-126), and its inverse, each rounded to nearest as a division
// rounds: a quotient by a number whose rounded inverse is known, corrected by its exact remainder, is
// the nearest one (Markstein's theorem), and so is an inverse after a step of Newton's from within a
// unit, but for divisors whose significand is all ones, where it depends on the hardware's first
// approximation.  Compared with the divisions for every finite float32, both are right on gfx950.
template <bool kE4M3>
__device__ __forceinline__ float scale_of(uint32_t largest, float *inverse) {
  constexpr float q = kE4M3 ? 448.f : 127.f, r = 1.f / q;
  const float most = __uint_as_float(largest);
  const float near = most * r;
  const float scale = fmaxf(fmaf(fmaf(-near, q, most), r, near), FLT_MIN);
  const float i0 = __builtin_amdgcn_rcpf(scale);
  *inverse = fmaf(fmaf(-scale, i0, 1.f), i0, i0);
  return scale;
}

// Four codes in a word.  (An integer's code is the low byte of the sum with 1.5 2^23, which rounds to
// the nearest integer, ties to even.)
template <bool kE4M3>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float inverse) {
#pragma clang fp contract(off)               // (the product is rounded before the sum)
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = x[e] * inverse;
  if constexpr (kE4M3) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(y[e] + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0C0C0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u),
                                 0x05040100u);
  }
}

template <typename T, int D, bool kE4M3, bool kRebind, int kShare>
__global__ __launch_bounds__(kWaves * kWave) void quant_write_kernel(const QuantWriteParams p) {
  constexpr int P = D / 2;
  constexpr int E = Store<T>::kPerChunk;
  constexpr int kLanes = P / E;              // lanes of a row, with E elements of each half
  constexpr int kTokens = kWave / kLanes;    // tokens of a wave
  constexpr int kRowBytes = D * static_cast<int>(sizeof(T)), kHalfBytes = kRowBytes / 2;
  const QuantStore &to = p.to;
  const int H = to.n_kv_heads;
  if constexpr (kRebind) {
    // The new lengths, and whether the offsets are those of total_k tokens, by the first workgroup
    // (also when there are none).
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
      for (int b = threadIdx.x; b < p.batch; b += kWaves * kWave) {
        const int s0 = p.sel_off[b], s1 = p.sel_off[b + 1];
        if (p.new_len != nullptr) p.new_len[b] = p.start[b] + (s1 - s0);
        const bool bad = s1 < s0 || (b == 0 && s0 != 0) || (b == p.batch - 1 && s1 != p.n_tok);
        if (bad && p.err != nullptr) atomicOr(p.err, PRCR_DERR_OFFSETS);
      }
  }
  __shared__ f32x4 s_angle[kWaves / kShare][E][kWave];   // of a lane's pairs (float32 rows: cos and sin as doubles)
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % kLanes;
  const int group = wave / kShare, member = wave % kShare;   // kShare waves share a group of tokens
  if (p.n_tok == 0) return;
  const int64_t t64 = (static_cast<int64_t>(blockIdx.x) * (kWaves / kShare) + group) * kTokens + lane / kLanes;
  const bool in_range = t64 < p.n_tok;
  const int t = in_range ? static_cast<int>(t64) : p.n_tok - 1;
  // The workgroup's rows; a wave takes every kShare-th.
  const int row_first = static_cast<int>(blockIdx.y) * p.rows_per_group, row1 = min(row_first + p.rows_per_group, p.rows);
  const int row0 = min(row_first + member, row1 - 1);
  const bool keys = blockIdx.z == 0;         // the workgroup's array
  const bool tells = in_range && c == 0 && blockIdx.y == 0 && keys && member == 0;   // the lane that reports for its token

  // The rows of one array, and of the slot's bases what to add for row r.
  const char *const rows_in = static_cast<const char *>(keys ? p.k : p.v) + c * 16;
  char *const codes = static_cast<char *>(keys ? to.k : to.v);
  float *const scales = keys ? to.k_scale : to.v_scale;
  struct Row {
    u32x4 lo, hi;
  };
  auto fetch = [&](int64_t source, int r) -> Row {
    const char *const row = rows_in + (source + r) * kRowBytes;
    return {load_nt(row), load_nt(row + kHalfBytes)};
  };
  auto offset = [&](int r, int64_t *scale) -> int64_t {
    const int l = kRebind ? static_cast<int>(p.by_heads.divide(static_cast<uint32_t>(r))) : p.layer;
    const int h = kRebind ? r - l * H : r;
    *scale = l * to.layer_scales + static_cast<int64_t>(h) * to.head_scales;
    return l * to.layer_rows + static_cast<int64_t>(h) * to.head_rows;
  };

  // The token: its sequence, position and slot, and its first row.  What the loads need is read in
  // as few dependent rounds as the data allow, from clamped places and outside branches (a load that
  // only a branch uses would move into it, a round trip later); the lanes without a token leave behind them.
  constexpr int kMine = E / kShare;          // angles that a thread computes: its lane's pairs member, member + kShare, ...
  double freq[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) freq[i] = p.inv_freq[c * E + member + i * kShare];
  int b, flag = 0;
  double pos[3];
  int64_t source;                            // index of the token's first row
  SlotEntry entry;
  Row first{};
  int64_t v_from = 0, v_from_scale = 0;      // of a memory without values: the slot's bases
  if constexpr (kRebind) {
    const int m = p.sel_idx[t];
#pragma unroll
    for (int a = 0; a < 3; ++a) pos[a] = p.new_pos[3 * static_cast<int64_t>(t) + a];
    // The last sequence that begins at or before t.  Fewer than 64 sequences' offsets are held by the
    // wave's lanes, one each; all lanes take part in every shuffle, whatever their own `at` is (one that
    // were switched off would be read as 0).
    int s0, s1, last = 0;
    if (p.batch < kWave) {
      const int held = p.sel_off[min(lane, p.batch)];
#pragma unroll
      for (int step = 32; step > 0; step >>= 1) {
        const int at = last + step, begins = __shfl(held, at & 63);
        last = at <= p.batch && begins <= t ? at : last;
      }
      b = min(last, p.batch - 1);
      s0 = __shfl(held, b);
      s1 = __shfl(held, b + 1);
    } else {
      int hi = p.batch;
      while (last < hi) {
        const int mid = (last + hi + 1) / 2;
        if (p.sel_off[mid] <= t) last = mid; else hi = mid - 1;
      }
      b = min(last, p.batch - 1);
      s0 = p.sel_off[b];
      s1 = p.sel_off[b + 1];
    }
    const bool offsets_ok = last < p.batch && s0 >= 0 && s0 <= t && t < s1 && s1 <= p.n_tok;
    const bool in_memory = m >= 0 && m < p.max_visual;
    source = (static_cast<int64_t>(b) * p.max_visual + (in_memory ? m : 0)) * p.rows;
    const bool copies = !keys && p.v_slot != nullptr;
    if (in_memory && !copies) first = fetch(source, row0);
    const int32_t n_visual = p.n_visual[b];
    const int64_t len = p.start[b];
    entry = entry_of_slot(to, b, len + (static_cast<int64_t>(t) - s0));
    flag = !offsets_ok ? PRCR_DERR_OFFSETS : (in_memory && m < n_visual ? 0 : PRCR_DERR_INDEX);
    if (p.v_slot != nullptr && flag == 0) {
      const int64_t vs = p.v_slot[static_cast<int64_t>(b) * p.max_visual + m];
      if (vs < 0 || vs >= len) {
        flag = PRCR_DERR_INDEX;
      } else {
        const Place from = place_of(to, b, entry_of_slot(to, b, vs));
        flag = from.flag;
        v_from = from.row;
        v_from_scale = from.scale;
      }
    }
  } else {
    b = static_cast<int>(p.by_seq.divide(static_cast<uint32_t>(t)));
    const int s = t - b * p.s_src;
    const int32_t n = p.n_tokens[b];
    const int64_t start = p.start[b];
#pragma unroll
    for (int a = 0; a < 3; ++a) pos[a] = p.pos[3 * static_cast<int64_t>(t) + a];
    entry = entry_of_slot(to, b, start + s);
    source = static_cast<int64_t>(t) * H;
    const bool live = in_range && s < n;
    if (live) first = fetch(source, row0);
    if ((n < 0 || n > p.s_src) && s == 0 && tells && p.err != nullptr) atomicOr(p.err, PRCR_DERR_INDEX);
    if (!live) flag = -1;                    // nothing to do
  }
  // The angles of the tokens, once for the workgroup.
  if (keys) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int pair = c * E + member + i * kShare;
      double sn, cs;
      turn((p.on_h >> pair & 1u ? pos[1] : p.on_w >> pair & 1u ? pos[2] : pos[0]) * freq[i], &sn, &cs);
      s_angle[group][member + i * kShare][lane] = sizeof(T) == 2 ? split_angle(cs, sn) : __builtin_bit_cast(f32x4, f64x2{cs, sn});
    }
    __syncthreads();
  }
  const Place at = place_of(to, b, entry);
  if (flag == 0) flag = at.flag;
  if (tells && flag >= 0) {
    if (flag != 0 && p.err != nullptr) atomicOr(p.err, flag);
    if (kRebind && p.slot_mapping != nullptr) p.slot_mapping[t] = flag == 0 ? at.id : -1;
  }
  if (flag != 0 || !in_range || row_first + member >= row1) return;

  const bool odd = c & 1;
  const int out_at = odd ? P + (c - 1) * E : c * E;
  // Quantises a row and stores it: 2 E codes a lane.  Of two neighbours, which hold E codes of each
  // half, the even lane stores both's of the first half and the odd lane both's of the second.
  auto put = [&](const Row &x, int r) {
    const uint32_t most = group_max<kLanes>(largest<T>(x.lo, x.hi));
    const uint32_t keep = most < 0x7F800000u ? ~0u : 0u;   // (a row with an infinity or a NaN: codes 0)
    float inverse;
    const float scale = scale_of<kE4M3>(most, &inverse);
    uint32_t w[E / 2];                       // the first half's words, then the second's
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      float y[4];
      elements<T>(x.lo, i, y);
      w[i] = encode4<kE4M3>(y, inverse) & keep;
      elements<T>(x.hi, i, y);
      w[E / 4 + i] = encode4<kE4M3>(y, inverse) & keep;
    }
    typedef uint32_t out_words __attribute__((ext_vector_type(E / 2)));
    out_words out;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const uint32_t mine = odd ? w[E / 4 + i] : w[i], other = odd ? w[i] : w[E / 4 + i];
      const uint32_t theirs = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(other), 0xB1, 0xF, 0xF, false));
      out[i] = odd ? theirs : mine;
      out[E / 4 + i] = odd ? mine : theirs;
    }
    int64_t scale_at;
    out_words *const to_row = reinterpret_cast<out_words *>(codes + (at.row + offset(r, &scale_at)) * D + out_at);
    __builtin_nontemporal_store(out, to_row);
    // (All of the row's lanes write it: behind a branch, the waits for loads would have to allow for its
    // not having been issued, and so wait for it.)
    scales[at.scale + scale_at] = keep != 0u ? scale : __uint_as_float(0x7FC00000u);
  };
  // kBatch rows at a time, all on their way before the first is made.  float32 rows of one layer are best one at
  // a time (8 prompts of 1,500 tokens, 8 heads: 20.8 us, by twos 22.0), bf16 rows two (2,560 tokens:
  // 25.4, one 29.9); revisited bf16 rows of 128 four (16 x 512 tokens in 28 layers: 142 us, by twos
  // 152), other ones two (64 features: 46.8, by fours 49.7).
  constexpr int kBatch = kRebind ? (sizeof(T) == 2 && D == 128 ? 4 : 2) : (sizeof(T) == 2 ? 2 : 1);
  auto go = [&](auto &&make) {
    for (int r = row0; r < row1; r += kBatch * kShare) {
      Row x[kBatch];
      x[0] = r > row0 ? fetch(source, r) : first;
#pragma unroll
      for (int i = 1; i < kBatch; ++i) x[i] = fetch(source, min(r + i * kShare, row1 - 1));
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (r + i * kShare >= row1) break;
        make(x[i]);
        put(x[i], r + i * kShare);
      }
    }
  };
  if (keys) {
    f32x4 angle[E];
#pragma unroll
    for (int e = 0; e < E; ++e) angle[e] = s_angle[group][e][lane];
    go([&](Row &x) {
      if constexpr (sizeof(T) == 2) {
        // (Or the doubles that turn_bf16 seldom needs would be made before the loop, and kept.)
#pragma unroll
        for (int e = 0; e < E; ++e) asm volatile("" : "+v"(angle[e]));
        turn_bf16(x.lo, x.hi, angle);
      } else {
        double cs[E], sn[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const f64x2 t = __builtin_bit_cast(f64x2, angle[e]);
          cs[e] = t[0];
          sn[e] = t[1];
        }
        const Row y = x;
        Store<T>::rotate(y.lo, y.hi, cs, sn, x.lo, x.hi);
      }
    });
  } else if (kRebind && p.v_slot != nullptr) {
    // (the slot's rows lie below the length, and so are none that this launch writes)
    for (int r = row0; r < row1; r += kShare) {
      int64_t scale_at;
      const int64_t row = offset(r, &scale_at);
      typedef uint32_t some_words __attribute__((ext_vector_type(E / 2)));
      *reinterpret_cast<some_words *>(codes + (at.row + row) * D + c * 2 * E) =
          *reinterpret_cast<const some_words *>(codes + (v_from + row) * D + c * 2 * E);
      scales[at.scale + scale_at] = scales[v_from_scale + scale_at];   // (all of the row's lanes: the same)
    }
  } else {
    go([](Row &) {});
  }
}

template <typename T, int D, bool kE4M3, bool kRebind, int kShare>
hipError_t launch_shared(const QuantWriteParams &in, int64_t per, hipStream_t stream) {
  QuantWriteParams p = in;
  constexpr int kTokens = kWaves / kShare * (kWave / (D / 2 / Store<T>::kPerChunk));   // of a workgroup
  while ((p.rows + per - 1) / per > 65535) per *= 2;
  p.rows_per_group = static_cast<int32_t>(std::min<int64_t>(per, p.rows));
  const int64_t blocks = std::max<int64_t>(1, (static_cast<int64_t>(p.n_tok) + kTokens - 1) / kTokens);
  if (!grid_fits(blocks, kWaves * kWave)) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>((p.rows + p.rows_per_group - 1) / p.rows_per_group), 2);
  quant_write_kernel<T, D, kE4M3, kRebind, kShare><<<grid, kWaves * kWave, 0, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int D, bool kE4M3, bool kRebind>
hipError_t launch(const QuantWriteParams &in, hipStream_t stream) {
  QuantWriteParams p = in;
  p.by_seq = Divisor::of(kRebind ? 1 : p.s_src);
  p.by_heads = Divisor::of(p.to.n_kv_heads);
  // Waves that share a group of tokens spread over them what is done once a token (half of a row's work), and of
  // the angles compute their share.  Few rows are the latency of one wave, shortest with the most waves; of many, a
  // wave has four.  Kernel times in us, bf16 rows of 128, one, two and four waves to a group, of 4 and of 8 heads:
  //       64 tokens    6.8   5.2   4.5      9.9   6.7   5.2
  //    2,000           8.1   6.1   5.0     12.0   8.2   6.0
  //    4,000           8.7   6.7   6.5     12.7   9.4   8.0
  //    8,000           9.6   8.6   9.7     14.7  12.9  14.5
  //   20,480          17.0  16.2  19.7     29.0  27.2  28.5
  // From 2,048 units on the rule gives 4 heads one wave and 8 heads two, where up to some 5,000 tokens twice as many
  // are faster: six ragged turns, 4,186 tokens in 6,558 rows, 4 heads, take 9.1 us so, 7.9 with two, 8.4 with four.
  // (That is not the padding: without it they take 8.7, and as many rows without a token 4.5.)
  //
  // A revisit's many rows are dealt to four waves, as many to each as leave a thousand waves an array, up to 28
  // (float32: 4).  4 x 64 tokens of 28 x 4 rows, with 2, 4, 8 and 28 a wave: 10.6, 8.2, 11.5 and 24.3 us, 4 x 256
  // tokens 29, 23.2, 20.5 and 27.8 (the rule: 4 and 14).  16 x 512 tokens, bf16 rows of 128, up to 4, 8, 16 and 28 a wave:
  //   28 x 4    149  138  132  128   (memories of 2,304 tokens and long caches, paged: 152, 139, 137, 137)
  //   36 x 8    366  337  339  343
  //   64 x 8    655  605  616  624
  //   13 x 5     98   89   86   80
  // and 32 x 64 tokens of 28 x 4 rows 41.6, 38.3, 39.0 and 39.1, paged 42.2, 38.8, 38.3 and 37.2.  float32, paged, up
  // to 4, 8 and 28: 28 x 4 rows 228, 231 and 242, 36 x 8 549, 570 and 590, 13 x 5 140, 143 and 145.
  constexpr int kGroup = kWave / (D / 2 / Store<T>::kPerChunk);
  const int64_t units = (static_cast<int64_t>(p.n_tok) + kGroup - 1) / kGroup * p.rows;   // a group of tokens' row
  if constexpr (kRebind) {
    const int64_t per = std::min<int64_t>(std::max<int64_t>((units / 1024 + 1) / 2 * 2, 2), sizeof(T) == 2 ? 28 : 4);
    return launch_shared<T, D, kE4M3, true, 4>(p, 4 * per, stream);
  } else {
    const int32_t share = units < 2048 ? p.rows : p.rows / 4;
    if (share < 2) return launch_shared<T, D, kE4M3, false, 1>(p, p.rows, stream);
    if (share < 4) return launch_shared<T, D, kE4M3, false, 2>(p, p.rows, stream);
    return launch_shared<T, D, kE4M3, false, 4>(p, p.rows, stream);
  }
}

template <typename T, int D, bool kRebind>
hipError_t dispatch_code(const QuantWriteParams &p, hipStream_t stream) {
  return p.to.code == PRCR_E4M3 ? launch<T, D, true, kRebind>(p, stream) : launch<T, D, false, kRebind>(p, stream);
}

template <bool kRebind>
hipError_t dispatch(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  if (dtype == PRCR_F32)
    return head_dim == 64 ? dispatch_code<float, 64, kRebind>(p, stream) : dispatch_code<float, 128, kRebind>(p, stream);
  return head_dim == 64 ? dispatch_code<uint16_t, 64, kRebind>(p, stream) : dispatch_code<uint16_t, 128, kRebind>(p, stream);
}

}  // namespace

hipError_t launch_quant_append(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dispatch<false>(p, dtype, head_dim, stream);
}
hipError_t launch_quant_rebind(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dispatch<true>(p, dtype, head_dim, stream);
}

}  // namespace prcr
