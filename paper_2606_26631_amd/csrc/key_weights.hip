// The weight each cached key received from the last tokens: for every sequence b, KV head h
// and slot j,
//   w[b][h][j] (+)= sum over the rows that see j, and the heads of group h, of exp(s_j - lse),
// s_j and lse as chunk attention has them.
//
// A workgroup takes a stretch of keys of one sequence and KV head, 32 kBlocks keys a wave, in
// registers, and runs through the rows that see them, 32 at a time, which all its waves
// read from LDS (two tiles of them, the next one's loads in flight).  The scores are formed as
// Q (32 rows) x K^T (32 keys), so that a lane holds 16 rows' scores of one key and adds
// their weights in its own registers: no other lane's, no atomics, a fixed order.
#include <algorithm>

#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kWaves = 4;
constexpr int kRows = 32;

__device__ __forceinline__ void load_to_lds(const char *from, char *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

template <typename T, int D, bool kPaged, int kBlocks>
__global__ __launch_bounds__(kWaves * kWave, 2) void key_weights_kernel(const AttendParams p) {
  constexpr bool kHalf = sizeof(T) == 2;
  constexpr int kRowBytes = D * static_cast<int>(sizeof(T));
  constexpr int kChunks = kRowBytes / 16;
  constexpr int kRowsPerLoad = kWave / kChunks;
  constexpr int kMine = kRows / kRowsPerLoad / kWaves;      // loads of a row tile per wave
  constexpr int kQ = kHalf ? D / 16 : D / 8;
  constexpr int kKeys = kWaves * 32 * kBlocks;
  static_assert(kMine >= 1, "a row tile is at least a load per wave");
  __shared__ __align__(1024) char s_q[2][kRows * kRowBytes];
  __shared__ float s_lse[2][kRows];
  __shared__ int s_limit[2][kRows];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane & 31, half = lane / 32;
  const uint32_t id = blockIdx.x;
  const uint32_t by_head = p.by_heads.divide(id);
  const int kvh = static_cast<int>(id - by_head * static_cast<uint32_t>(p.n_kv_heads));
  const int b = static_cast<int>(p.by_split.divide(by_head));     // (n_split: key stretches per sequence)
  const int k0 = (static_cast<int>(by_head) - b * p.n_split) * kKeys;
  const int32_t len = clamp_length(p.cache_len[b], p.capacity);
  float *const weights = p.weights + (static_cast<int64_t>(b) * p.n_kv_heads + kvh) * p.capacity;
  if (k0 >= len) {
    if (!p.accumulate)
      for (int j = k0 + threadIdx.x; j < min(k0 + kKeys, p.capacity); j += kWaves * kWave) weights[j] = 0.f;
    return;
  }
  const Rows rows = rows_of(p, b);
  const int G = p.group, first = len - rows.n;
  const int from = max(p.window > 0 ? max(rows.n - p.window, 0) : 0, k0 - first);   // first token that counts
  const int row0 = min(from, rows.n) * G, n_rows = rows.n * G;

  // The wave's keys: bf16, of product i, elements 16 i + 8 half + 0..7; float32, the lane's
  // half of the row.
  const int kw = k0 + wave * 32 * kBlocks;
  u32x4 k[kBlocks][kQ];
  bool live[kBlocks];
  bool bad_block = false;
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb) {
    const int j = min(kw + 32 * kb + l32, len - 1);
    int64_t row;
    live[kb] = kw + 32 * kb + l32 < len;
    if constexpr (kPaged) {
      const int lb = p.block_shift >= 0 ? j >> p.block_shift : j / p.block_size;
      const int32_t blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + lb];
      const bool ok = blk >= 0 && blk < p.n_blocks;
      bad_block |= live[kb] && !ok;
      live[kb] = live[kb] && ok;
      row = ((static_cast<int64_t>(p.layer) * p.n_blocks + (ok ? blk : 0)) * p.block_size + (ok ? j - lb * p.block_size : 0)) *
                p.n_kv_heads + kvh;
    } else {
      row = ((static_cast<int64_t>(b) * p.n_layers + p.layer) * p.n_kv_heads + kvh) * p.s_max + j;
    }
    const char *const at = static_cast<const char *>(p.cache_k) + row * kRowBytes;
#pragma unroll
    for (int i = 0; i < kQ; ++i)
      k[kb][i] = load_nt(at + (kHalf ? 2 * i + half : half * kQ + i) * 16);
  }
  if (kPaged && p.err != nullptr && __any(bad_block) && lane == 0) atomicOr(p.err, PRCR_DERR_BLOCK);

  auto token_of = [&](int r) -> int { return static_cast<int>(p.by_group.divide(static_cast<uint32_t>(r))); };
  auto row_index = [&](int r, int token) -> int64_t {
    return (static_cast<int64_t>(rows.start) + token) * p.n_q_heads + kvh * G + (r - token * G);
  };
  const int in_load = lane / kChunks, chunk = lane % kChunks;
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
  // Of row `threadIdx.x` of a tile: what is taken from its scores, and the last slot it sees.
  // Rows past the last one, and rows that see nothing, give no weight.
  float lse = 0.f;
  int limit = 0;
  auto load_lse = [&](int r0) {
    const int r = min(r0 + static_cast<int>(threadIdx.x), n_rows - 1);
    const int token = token_of(r);
    limit = first + token;
    lse = p.lse[row_index(r, token)];
    if (r0 + static_cast<int>(threadIdx.x) >= n_rows || limit < 0) lse = __builtin_inff();
  };

  double w[kBlocks] = {};                    // (the first keys add up every row there is: float32 lost 1e-6 of 10,000)
  int buf = 0;
  if (row0 < n_rows) {
    load_rows(row0, s_q[0]);
    if (threadIdx.x < kRows) {
      load_lse(row0);
      s_lse[0][threadIdx.x] = lse;
      s_limit[0][threadIdx.x] = limit;
    }
  }
  for (int r0 = row0; r0 < n_rows; r0 += kRows, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const bool more = r0 + kRows < n_rows;
    if (more) {
      load_rows(r0 + kRows, s_q[buf ^ 1]);
      if (threadIdx.x < kRows) load_lse(r0 + kRows);
    }
    const char *const qrow = s_q[buf] + l32 * kRowBytes;
    const int sw = l32 & (kChunks - 1);
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
    f32x4 off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) off[i] = *reinterpret_cast<const f32x4 *>(&s_lse[buf][8 * i + 4 * half]);
    const bool masked = kw + 32 * kBlocks - 1 > first + token_of(r0);
    float sum[kBlocks] = {};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int last = masked ? s_limit[buf][8 * (i / 4) + 4 * half + i % 4] : INT32_MAX;
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) {
        const float e = exp2_hw(fmaf(s[kb][i], p.scale, -off[i / 4][i % 4]) * 1.44269504088896341f);
        sum[kb] += kw + 32 * kb + l32 <= last ? e : 0.f;
      }
    }
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) w[kb] += static_cast<double>(sum[kb]);
    if (more && threadIdx.x < kRows) {
      s_lse[buf ^ 1][threadIdx.x] = lse;
      s_limit[buf ^ 1][threadIdx.x] = limit;
    }
  }
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb) {
    const float sum = static_cast<float>(w[kb] + __shfl_xor(w[kb], 32));
    const int j = kw + 32 * kb + l32;
    if (half != 0 || j >= p.capacity) continue;
    if (p.accumulate) {
      if (live[kb]) weights[j] += sum;
    } else {
      weights[j] = live[kb] ? sum : 0.f;
    }
  }
}

template <typename T, int D, bool kPaged, int kBlocks>
hipError_t weigh(const AttendParams &in, hipStream_t stream) {
  AttendParams p = in;
  p.n_split = (p.capacity + kWaves * 32 * kBlocks - 1) / (kWaves * 32 * kBlocks);
  p.by_split = Divisor::of(p.n_split);
  const int64_t blocks = static_cast<int64_t>(p.n_kv_heads) * p.n_split * p.batch;
  if (blocks > INT32_MAX || !grid_fits(blocks, kWaves * kWave)) return hipErrorInvalidConfiguration;
  key_weights_kernel<T, D, kPaged, kBlocks><<<static_cast<unsigned>(blocks), kWaves * kWave, 0, stream>>>(p);
  return hipGetLastError();
}

template <typename T, bool kPaged>
hipError_t weigh_dim(const AttendParams &p, int head_dim, hipStream_t stream) {
  if constexpr (sizeof(T) == 4)
    return head_dim == 64 ? weigh<T, 64, kPaged, 1>(p, stream) : weigh<T, 128, kPaged, 1>(p, stream);
  return head_dim == 64 ? weigh<T, 64, kPaged, 2>(p, stream) : weigh<T, 128, kPaged, 2>(p, stream);
}

}  // namespace

hipError_t launch_key_weights(const AttendParams &p, prcr_dtype dtype, int head_dim, bool paged, hipStream_t stream) {
  if (dtype == PRCR_F32)
    return paged ? weigh_dim<float, true>(p, head_dim, stream) : weigh_dim<float, false>(p, head_dim, stream);
  return paged ? weigh_dim<uint16_t, true>(p, head_dim, stream) : weigh_dim<uint16_t, false>(p, head_dim, stream);
}

}  // namespace prcr
