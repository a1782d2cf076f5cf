// What the kernels of decode attention share, over caches in the model's type and in 8 bits: how
// sequences and keys are dealt to workgroups, the end of a workgroup's chunk, and the exact
// bf16 operands of float32 numbers.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "prcr_internal.h"
#include "rotary.h"

namespace prcr {

// The merge of a call's partials (decode.hip), by decode_combine_kernel.
hipError_t launch_decode_merge(const DecodeParams &p, int head_dim, bool paged, hipStream_t stream);

namespace {

constexpr int kUnits = 256;  // compute units of the chip

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The first splits of `pairs` (sequence, KV head) pairs for lo to hi workgroups that fill whole rounds over
// the chip to the share `enough`, or else the nearest; at most `room` (a search of at most some tens
// of steps, on every call).
inline int64_t splits_in_rounds(int64_t pairs, int64_t lo, int64_t hi, int64_t room, double enough) {
  int64_t best = ceil_div(lo, pairs);
  double share = 0;
  for (int64_t n = best; n <= std::min(ceil_div(hi, pairs), room) && share < enough; ++n) {
    const double s = static_cast<double>(pairs * n) / static_cast<double>(ceil_div(pairs * n, kUnits) * kUnits);
    if (s > share + 1e-9) {
      share = s;
      best = n;
    }
  }
  return std::min(best, room);
}

// Scores are kept in base-2 units (the query carries log2(e)), so every
// softmax weight is one hardware exp2.
constexpr double kLog2e = 1.4426950408889634;
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Lane permutation within a 16-lane DPP row (no LDS round trip).
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xF, 0xF, false));
}

// Sum over the LPK consecutive lanes that hold one key row.  Every lane of the
// group ends with the same total: partners add the same two values at each step.
template <int LPK>
__device__ __forceinline__ float group_sum(float s) {
  static_assert(LPK == 16 || LPK == 32, "unsupported lane group");
  s += dpp<0xB1>(s);                               // quad permutation 1,0,3,2: lane ^ 1
  s += dpp<0x4E>(s);                               // quad permutation 2,3,0,1: lane ^ 2
  s += dpp<0x141>(s);                              // mirror in 8-lane halves: the other quad
  s += dpp<0x140>(s);                              // mirror in the 16-lane row: the other half
  if constexpr (LPK >= 32) s += __shfl_xor(s, 16);
  return s;
}

// Workgroup barrier that orders LDS accesses only: loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Sequence taken by workgroup row z, and its length entry.  With at most 64 sequences
// (lane l reads length l), the rows go to the sequences in order of decreasing length,
// ties by index.  Workgroups are dealt to the compute units in turn, so that each unit
// then holds chunks of long and of short sequences rather than a random mix: on a
// paged batch of 2,918-6,424 keys this measured 6 % faster.  Results do not depend
// on the order (each sequence is computed the same way by whichever row takes it).
//
// Every workgroup does this before its first key, so its waves share the work: a lane's
// rank is the number of keys (length, then lower index) above its own, and wave w counts
// among sequences 16 w to 16 w + 15.  With 64 sequences every wave counting all of them
// took 2.7 us (two compares each) or 1.1 us (one); the shared count takes 0.6.
template <int kWaves>
__device__ __forceinline__ int sequence_of_row(const DecodeParams &p, int lane, int z, int *len) {
  if (p.batch > kWave) {
    *len = p.cache_len[z];
    return z;
  }
  constexpr int kShare = kWave / kWaves;     // sequences a wave counts
  const int raw = lane < p.batch ? p.cache_len[lane] : 0;
  if (p.batch == 1) {
    *len = __builtin_amdgcn_readfirstlane(raw);
    return 0;
  }
  // Order of the lengths as one number: those above 2^25 - 1 count as equal.
  const uint32_t mine = lane < p.batch ? (static_cast<uint32_t>(min(max(raw, 0), (1 << 25) - 1)) << 6 | (63 - lane)) + 1 : 0;
  auto above = [&](int i0, int n) -> int {
    int count = 0;
#pragma unroll
    for (int i = 0; i < n; ++i)
      count += static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(mine), i0 + i)) > mine ? 1 : 0;
    return count;
  };
  int rank = 0;
  if (p.batch <= kShare) {
    for (int i0 = 0; i0 < p.batch; i0 += 4) rank += above(i0, 4);
  } else {
    __shared__ int s_rank[kWaves][kWave];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    s_rank[wave][lane] = above(wave * kShare, kShare);
    lds_barrier();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) rank += s_rank[w][lane];
  }
  const unsigned long long hit = __ballot(lane < p.batch && rank == z);
  const int b = __builtin_amdgcn_readfirstlane(hit ? __ffsll(static_cast<long long>(hit)) - 1 : z);
  *len = __builtin_amdgcn_readlane(raw, b);
  return b;
}

// The bf16 kernel's grid is (KV head, row, split): the first workgroups to be placed are the
// first chunks of all sequences, and the ones without keys come last.  (With the splits
// innermost, the workgroups with keys of a sequence of 4,000 in a cache of 63 splits shared
// every second compute unit: 11.1 us a layer, now 9.3.)  Every second round of workgroups over
// the chip takes the rows in reverse, so that a compute unit's second workgroup
// is short where its first is long: two layers of 64 paged sequences of 2,912-6,512 keys
// in two splits took 230.0 us with the splits innermost, 243.2 with the rows in the same
// order in both splits and 215.7 this way.  The float32 kernel has three rounds, and is
// faster with the splits innermost (238.8 against 257.3 us, 32 such sequences, 4 heads).
__device__ __forceinline__ int row_of(const DecodeParams &p, int split, int y) {
  const uint32_t before = static_cast<uint32_t>(split) * gridDim.x * gridDim.y;   // workgroups of earlier splits
  return before / kUnits & 1 ? p.batch - 1 - y : y;
}

// Keys per workgroup of a sequence of len keys: an even share of its n_split workgroups,
// in whole rounds of p.round keys, so that no workgroup of a sequence waits on a longer
// one; no fewer than p.min_keys where p.fill workgroups would do (plan_splits).
// Workgroups past the sequence's last key have nothing to do and write nothing (with
// p.all_splits: an empty partial).
__device__ __forceinline__ int chunk_keys(const DecodeParams &p, int len) {
  // ceil(len / n) by the launcher's ceil(2^32 / n): one too many at most (len < 2^30).
  auto share = [&](int n, uint32_t inverse) -> int {
    return n == 1 ? len : static_cast<int>(__umulhi(static_cast<uint32_t>(len + n - 1), inverse));
  };
  int per = share(p.n_split, p.split_inverse);
  if (p.n_split > p.fill && per < p.min_keys) per = share(p.fill, p.fill_inverse);
  return (per + p.round - 1) & -p.round;   // (a power of two)
}

// Length of a sequence as the kernels use it: within [0, capacity].
__device__ __forceinline__ int clamp_len(const DecodeParams &p, bool paged, int len) {
  const int64_t cap = paged ? static_cast<int64_t>(p.max_blocks) * p.block_size : p.s_max;
  return static_cast<int>(min(max(static_cast<int64_t>(len), int64_t{0}), cap));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));   // at any float

// Ends a chunk of kWaves waves (`thread` among them): merges the waves' running maxima, sums of weights and weighted
// values (a head's value is the sum of kParts rows, kStep rows apart) and writes them to the
// workspace for decode_combine_kernel, or, where every sequence is one chunk (p.direct), to
// the output at once.  Four features of one head per thread, every LDS read issued before
// the first use; a feature at a time this took 0.6 us of the 4 us that a short chunk takes.
template <int kWaves, int D, int GT, int kParts, int kStep, int kRows>
__device__ __forceinline__ void finish_split(const DecodeParams &p, int b, int kvh, int G, int split, int thread,
                                             const float (&s_m)[kWaves][GT], const float (&s_l)[kWaves][GT],
                                             const float (&s_o)[kWaves][kRows][D]) {
  const int64_t head0 = static_cast<int64_t>(b) * p.n_q_heads + kvh * G;
#pragma unroll
  for (int u = 0; u < (GT * D / 4 + kWaves * kWave - 1) / (kWaves * kWave); ++u) {
    const int idx = u * kWaves * kWave + thread;
    const int g = idx / (D / 4), d = idx % (D / 4) * 4;
    if (g >= G) break;
    float m[kWaves], l[kWaves];
    f32x4 o[kWaves][kParts];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      m[w] = s_m[w][g];
      l[w] = s_l[w][g];
#pragma unroll
      for (int q = 0; q < kParts; ++q) o[w][q] = *reinterpret_cast<const f32x4 *>(&s_o[w][q * kStep + g][d]);
    }
    float M = -FLT_MAX, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, m[w]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = exp2_fast(m[w] - M);
      L += l[w] * wt;
      f32x4 v = o[w][0];
#pragma unroll
      for (int q = 1; q < kParts; ++q) v += o[w][q];
      O += v * wt;
    }
    if (p.direct) {
#pragma unroll
      for (int e = 0; e < 4; ++e) O[e] = L != 0.f ? O[e] / L : 0.f;   // (a NaN stays one)
      *reinterpret_cast<f32x4_any *>(p.out + (head0 + g) * D + d) = O;
    } else {
      float *ws = p.ws + ((head0 + g) * p.n_split + split) * (D + 2);
      *reinterpret_cast<f32x4_any *>(ws + d) = O;
      if (d == 0) {
        ws[D] = M;
        ws[D + 1] = L;
      }
    }
  }
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma_16x16x32(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Orders this wave's LDS writes before its later LDS reads (LDS operations of a
// wave complete in issue order; this keeps the compiler from moving them).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Part `part` (0, 1, 2) of the three-way bf16 split of x, as bf16 bits in the
// upper half of a word.  Each part is the truncation of what the previous parts
// left, and every difference is exact in float32, so the parts sum to x.
__device__ __forceinline__ uint32_t split_part(float x, int part) {
  const uint32_t hi = __float_as_uint(x) & 0xFFFF0000u;
  const float r1 = x - __uint_as_float(hi);
  const uint32_t mid = __float_as_uint(r1) & 0xFFFF0000u;
  const float r2 = r1 - __uint_as_float(mid);
  return part == 0 ? hi : (part == 1 ? mid : __float_as_uint(r2));
}

// Maximum over the 16 lanes of a DPP row; every lane of the row ends with it.
__device__ __forceinline__ float row_max16(float s) {
  s = fmaxf(s, dpp<0xB1>(s));
  s = fmaxf(s, dpp<0x4E>(s));
  s = fmaxf(s, dpp<0x141>(s));
  s = fmaxf(s, dpp<0x140>(s));
  return s;
}

// Upper halves of two words (a's in the low half of the result), and lower halves.
__device__ __forceinline__ uint32_t pack_hi(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
__device__ __forceinline__ uint32_t pack_lo(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// Exchanges lanes 8..15 of each row of 16 in a with lanes 0..7 of the row in b.
__device__ __forceinline__ void swap_rows8(u32x4 &a, u32x4 &b) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int x = static_cast<int>(a[w]), y = static_cast<int>(b[w]);
    a[w] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false));
    b[w] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false));
  }
}

constexpr int kTile = 32;   // keys per wave and tile: the value product's contraction length

}  // namespace
}  // namespace prcr
