// Shared by the operators on several tokens per sequence: chunk attention, the keys'
// weights and eviction.  Parameter blocks, launchers, and the device side of the packed
// query rows and of a cache row's address.
#pragma once

#include <cfloat>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "prcr_internal.h"
#ifdef __HIPCC__
#include "rotary.h"
#endif

namespace prcr {

// Packed query rows and the cache they look at.  Query row t of total_q is a token; a
// sequence's rows are q_off[b] .. q_off[b + 1] - 1, or the first q_len[b] of them.
struct AttendParams {
  const void *q;                  // [total_q][n_q_heads][head_dim], as given
  void *rotated;                  // weights: the same, rotated (workspace)
  const int32_t *q_off;           // [batch + 1]
  const int32_t *q_len;           // [batch] or null
  const int32_t *q_pos;           // [total_q][3]
  const int32_t *cache_len;       // [batch]
  const void *cache_k;
  const void *cache_v;
  const int32_t *block_table;
  void *out;                      // chunk attention: [total_q][n_q_heads][head_dim]
  float *lse;                     // [total_q][n_q_heads]: out (or null), or the weights' input
  float *part;                    // chunk attention: [total_q][n_q_heads][n_split][head_dim + 2];
                                  // weights: [n_split][batch][n_kv_heads][capacity]
  float *weights;                 // weights: [batch][n_kv_heads][capacity]
  int32_t *err;
  int32_t total_q, batch, n_layers, n_kv_heads, n_q_heads, group, layer;
  int32_t s_max, block_size, max_blocks, n_blocks;
  int32_t block_shift;            // log2(block_size) if a power of two, else -1
  int32_t capacity;               // slots per sequence: s_max, or max_blocks * block_size
  int32_t n_slots, n_split;       // chunk attention: row tiles there is room for, key splits;
                                  // weights: key stretches of a sequence, row splits (launcher)
  int32_t window;                 // weights: the last rows of each sequence that count (0: all)
  int32_t accumulate;
  float scale2;                   // |scale| log2(e)
  int32_t negate;                 // a negative scale: the rotated queries' sign is turned
  Divisor by_group, by_heads, by_split, by_slot, by_row;
  int8_t axis[kMaxPairs];
  double inv_freq[kMaxPairs];
};

struct EvictParams {
  const int32_t *cache_len;
  const float *weights;           // [batch][n_kv_heads][capacity]
  void *cache_k;
  void *cache_v;
  const int32_t *block_table;
  int32_t *new_len;               // [batch]
  int32_t *kept;                  // [batch][budget]
  float *new_weights;             // [batch][n_kv_heads][capacity] or null
  int32_t *v_slot;                // [batch][max_visual] of a key-only memory, or null
  float *score;                   // workspace [batch][capacity]: the scores' order as integers
  int32_t *first_moved;           // workspace [batch]: the first kept slot that moves
  uint32_t __attribute__((ext_vector_type(2))) *moves;   // workspace, paged: [batch][budget] pool slots, from and to
  int32_t *err;
  int32_t batch, n_layers, n_kv_heads, row_bytes;
  int32_t s_max, block_size, max_blocks, n_blocks, capacity;
  int32_t budget, keep_first, keep_last, max_visual;
};

// What a call of chunk attention needs besides its arguments: how its rows and keys are
// divided, and the bytes of its workspace (partial results of several splits).
struct ChunkPlan {
  bool few;                       // tiles of 32 rows, whose keys the waves share out (or of 128)
  int32_t n_slots, n_split;
  size_t bytes;
};
ChunkPlan plan_chunk(int64_t capacity, int32_t batch, int32_t total_q, int32_t n_q_heads, int32_t n_kv_heads,
                     int32_t head_dim);

// The same of the keys' weights (rotated queries, then partial sums): 32-key blocks a wave
// holds, key stretches of a sequence, and the workgroups that share a stretch's rows.
struct WeightsPlan {
  int32_t blocks, n_stretches, n_split;
  size_t rotated_bytes, bytes;
};
WeightsPlan plan_key_weights(int64_t capacity, int32_t batch, int32_t total_q, int32_t n_q_heads, int32_t n_kv_heads,
                             int32_t head_dim, int32_t window, prcr_dtype dtype);

// The report that the rotation and chunk attention begin with, by itself: for the keys' weights of a call
// without rows.
hipError_t launch_report(const AttendParams &p, hipStream_t stream);
hipError_t launch_rotate(const AttendParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream);
hipError_t launch_chunk(const AttendParams &p, const ChunkPlan &plan, prcr_dtype dtype, int head_dim, bool paged,
                        hipStream_t stream);
hipError_t launch_key_weights(const AttendParams &p, const WeightsPlan &plan, prcr_dtype dtype, int head_dim, bool paged,
                              hipStream_t stream);
hipError_t launch_evict(const EvictParams &p, bool paged, hipStream_t stream);

#ifdef __HIPCC__
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The rows of sequence b: its first row and their count (0 where the offsets are malformed),
// and whether they are.
struct Rows {
  int32_t start, n;
  bool bad;
};
__device__ __forceinline__ Rows rows_of(const AttendParams &p, int b) {
  const int32_t s = p.q_off[b], e = p.q_off[b + 1];
  Rows r{s, e - s, s < 0 || e < s || e > p.total_q};
  if (p.q_len != nullptr && !r.bad) {
    const int32_t n = p.q_len[b];
    r.bad = n < 0 || n > r.n;
    r.n = n;
  }
  if (r.bad) r.n = 0;
  return r;
}

__device__ __forceinline__ int32_t clamp_length(int32_t len, int32_t capacity) { return min(max(len, 0), capacity); }

// The larger of each lane's value and that of the lane 32 away.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor(x, d));
  return half_max(x);
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) x += __shfl_xor(x, d);
  return half_sum(x);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {   // to nearest, ties to even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// sin and cos of an angle, to about 2^-52.  The angle less the
// nearest multiple of pi/2 (kept as two doubles, one fused multiply-add each: Cody and Waite's
// reduction), then the Taylor series on [-pi/4, pi/4]; its terms of degree 17 and 18 are below
// 2^-54.  The math library's sincos, made for any double, took 10 us in a launch of a few waves.
__device__ __forceinline__ void turn(double x, double *sn, double *cs) {
  const double n = rint(x * 0.63661977236758134308);
  const double r = fma(-n, 6.12323399573676603587e-17, fma(-n, 1.57079632679489655800, x));
  const double z = r * r;
  double s = -1. / 1307674368000., c = 1. / 20922789888000.;
  s = fma(s, z, 1. / 6227020800.);
  c = fma(c, z, -1. / 87178291200.);
  s = fma(s, z, -1. / 39916800.);
  c = fma(c, z, 1. / 479001600.);
  s = fma(s, z, 1. / 362880.);
  c = fma(c, z, -1. / 3628800.);
  s = fma(s, z, -1. / 5040.);
  c = fma(c, z, 1. / 40320.);
  s = fma(s, z, 1. / 120.);
  c = fma(c, z, -1. / 720.);
  s = fma(s, z, -1. / 6.);
  c = fma(c, z, 1. / 24.);
  s = fma(s * z, r, r);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.);
  const int q = static_cast<int>(fma(-4., floor(n * 0.25), n));   // n modulo 4
  const double a = q & 1 ? c : s, b = q & 1 ? s : c;
  *sn = q & 2 ? -a : a;
  *cs = (q + 1) & 2 ? -b : b;
}

// A cosine and a sine as two floats each: cos high, cos low, sin high, sin low.
__device__ __forceinline__ f32x4 split_angle(double cs, double sn) {
  const float c = static_cast<float>(cs), s = static_cast<float>(sn);
  return f32x4{c, static_cast<float>(cs - static_cast<double>(c)), s, static_cast<float>(sn - static_cast<double>(s))};
}

// One pair of 16-byte chunks of bf16 rows, turned and rounded once to bf16.  The
// angles are split as above, exact to 2^-49.  In float32 with the
// products' errors kept, the result is within one unit of float32 of the exact one, so its
// rounding to bf16 is that of the exact one unless it lies that near to the middle of two bf16
// numbers; a chunk with such an element (some lane's, in one of ten) is done again in double.
// In double throughout this took 5,900 cycles a wave, the conversions most of it; it takes 3,900.
__device__ __forceinline__ void turn_bf16(u32x4 &lo, u32x4 &hi, const f32x4 (&angle)[8]) {
  u32x4 a, b;
  uint32_t nearest = ~0u;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float y[2][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float x = __uint_as_float(e ? lo[q] & 0xFFFF0000u : lo[q] << 16);
      const float z = __uint_as_float(e ? hi[q] & 0xFFFF0000u : hi[q] << 16);
      const f32x4 t = angle[2 * q + e];      // cos high, cos low, sin high, sin low
      const float zs = z * t[2], xs = x * t[2];
      const float ezs = fmaf(z, t[2], -zs), exs = fmaf(x, t[2], -xs);
      y[0][e] = fmaf(x, t[0], -zs) + fmaf(x, t[1], -fmaf(z, t[3], ezs));   // x cos - z sin
      y[1][e] = fmaf(z, t[0], xs) + fmaf(z, t[1], fmaf(x, t[3], exs));     // z cos + x sin
#pragma unroll
      for (int h = 0; h < 2; ++h)
        nearest = min(nearest, (__float_as_uint(y[h][e]) - 0x7FFEu) & 0xFFFFu);
    }
    a[q] = pack_bf16(y[0][0], y[0][1]);
    b[q] = pack_bf16(y[1][0], y[1][1]);
  }
  if (__any(nearest <= 4u)) {
    double cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = static_cast<double>(angle[e][0]) + static_cast<double>(angle[e][1]);
      sn[e] = static_cast<double>(angle[e][2]) + static_cast<double>(angle[e][3]);
    }
    Store<uint16_t>::rotate(lo, hi, cs, sn, a, b);
  }
  lo = a;
  hi = b;
}

// Reports what is wrong with the offsets and lengths, which the kernels only skip.
__device__ __forceinline__ void report(const AttendParams &p, int thread, int threads) {
  int bits = 0;
  for (int b = thread; b < p.batch; b += threads) {
    if (rows_of(p, b).bad) bits |= PRCR_DERR_OFFSETS;
    const int32_t len = p.cache_len[b];
    if (len != clamp_length(len, p.capacity)) bits |= PRCR_DERR_CAPACITY;
  }
  if (bits != 0) atomicOr(p.err, bits);
}

}  // namespace
#endif

}  // namespace prcr
