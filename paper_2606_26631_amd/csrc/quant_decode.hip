// Decode attention over the decoder cache in 8 bits (Eq. (14), as decode.hip has it): for each
// sequence and query head, with q' the query turned at its position times scale log2(e), in float32,
//   s_j = kscale_j (q' . kcode_j),   out = sum_j 2^(s_j - m) vscale_j vcode_j / sum_j 2^(s_j - m)
// over the slots below the sequence's length.  Split-K as there: one workgroup per key chunk, KV
// head and sequence, and the same merge of the chunks' partials.
#include <algorithm>

#include "decode_split.h"
#include "quant.h"

namespace prcr {
namespace {

constexpr int kWaves = 4;

template <int D, int GT, bool kPaged, bool kE4M3>
__global__ __launch_bounds__(kWaves * kWave) void quant_decode_kernel(const QuantDecodeParams p) {
  constexpr int E = 8;                       // codes of a lane
  constexpr int kLanes = D / E;              // lanes per key row
  constexpr int KPW = kWave / kLanes;        // keys per wave and step
  constexpr int KPB = kWaves * KPW;
  constexpr int P = D / 2;
  __shared__ float s_m[kWaves][GT];
  __shared__ float s_l[kWaves][GT];
  __shared__ __align__(16) float s_o[kWaves][GT][D];
  const int split = blockIdx.x, kvh = blockIdx.y;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int len_in;
  const int b = sequence_of_row<kWaves>(p, lane, blockIdx.z, &len_in);
  const int kg = lane / kLanes, c = lane % kLanes;
  const int G = p.group;
  const int len = clamp_len(p, kPaged, len_in);
  if (len != len_in && split == 0 && kvh == 0 && threadIdx.x == 0 && p.err != nullptr)
    atomicOr(p.err, PRCR_DERR_CAPACITY);
  const int chunk = chunk_keys(p, len);
  const int j0 = static_cast<int>(min(static_cast<int64_t>(len), static_cast<int64_t>(split) * chunk));
  const int j1 = static_cast<int>(min(static_cast<int64_t>(len), static_cast<int64_t>(j0) + chunk));
  if (j0 >= j1 && split > 0) return;

  float qv[GT][E];
  {
    const double pq = static_cast<double>(p.q_pos[b]), qs = static_cast<double>(p.scale) * kLog2e;
    const bool first = c < kLanes / 2;
    double cs[E], sn[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sincos(pq * p.inv_freq[(c * E + e) % P], &sn[e], &cs[e]);
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      const int64_t row = (static_cast<int64_t>(b) * p.n_q_heads + kvh * G + (g < G ? g : 0)) * D;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = c * E + e, j = first ? i + P : i - P;
        auto at = [&](int k) -> double {
          if (p.q_f32) return static_cast<const float *>(p.q)[row + k];
          return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(p.q)[row + k]) << 16);
        };
        const double y = first ? at(i) * cs[e] - at(j) * sn[e] : at(i) * cs[e] + at(j) * sn[e];
        qv[g][e] = static_cast<float>(y * qs);
      }
    }
  }
  float m[GT], l[GT], o[GT][E];
#pragma unroll
  for (int g = 0; g < GT; ++g) {
    m[g] = -FLT_MAX;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[g][e] = 0.f;
  }
  int bad_block = 0;
  for (int jb = j0; jb < j1; jb += KPB) {
    const int j = jb + wave * KPW + kg;
    bool live = j < j1;
    const int js = live ? j : j0;
    int64_t row, at;
    if constexpr (kPaged) {
      const int lb = js / p.block_size, off = js - lb * p.block_size;
      const int32_t blk = p.block_table[static_cast<int64_t>(b) * p.max_blocks + lb];
      const bool ok = blk >= 0 && blk < p.n_blocks;
      bad_block |= live && !ok;
      live = live && ok;
      const int64_t in = static_cast<int64_t>(p.layer) * p.n_blocks + (ok ? blk : 0);
      row = (in * p.block_size + off) * p.n_kv_heads + kvh;
      at = (in * p.n_kv_heads + kvh) * p.block_size + off;
    } else {
      row = at = ((static_cast<int64_t>(b) * p.n_layers + p.layer) * p.n_kv_heads + kvh) * p.s_max + js;
    }
    const uint32_t *const kr = reinterpret_cast<const uint32_t *>(static_cast<const char *>(p.cache_k) + row * D + c * E);
    const uint32_t *const vr = reinterpret_cast<const uint32_t *>(static_cast<const char *>(p.cache_v) + row * D + c * E);
    float k[E], v[E];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      decode4(kr[i], kE4M3, k + 4 * i);
      decode4(vr[i], kE4M3, v + 4 * i);
    }
    const float ks = p.k_scale[at], vs = p.v_scale[at];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(qv[g][e], k[e], s);
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) s += __shfl_xor(s, d);
      s *= ks;
      const float mn = live ? fmaxf(m[g], s) : m[g];
      const float corr = exp2_fast(m[g] - mn), w = live ? exp2_fast(s - mn) : 0.f;
      m[g] = mn;
      l[g] = l[g] * corr + w;
      const float wv = live ? w * vs : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = fmaf(wv, v[e], o[g][e] * corr);
    }
  }
  if (bad_block && p.err != nullptr) atomicOr(p.err, PRCR_DERR_BLOCK);
#pragma unroll
  for (int off = kLanes; off < kWave; off <<= 1) {
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      const float m2 = __shfl_xor(m[g], off), l2 = __shfl_xor(l[g], off), mx = fmaxf(m[g], m2);
      const float w1 = exp2_fast(m[g] - mx), w2 = exp2_fast(m2 - mx);
      l[g] = l[g] * w1 + l2 * w2;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = o[g][e] * w1 + __shfl_xor(o[g][e], off) * w2;
      m[g] = mx;
    }
  }
  if (kg == 0) {
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      if (c == 0) {
        s_m[wave][g] = m[g];
        s_l[wave][g] = l[g];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) s_o[wave][g][c * E + e] = o[g][e];
    }
  }
  __syncthreads();
  finish_split<kWaves, D, GT, 1, 1>(p, b, kvh, G, split, s_m, s_l, s_o);
}

template <int D, int GT, bool kPaged>
void launch_one(QuantDecodeParams p, prcr_code code, hipStream_t stream) {
  p.round = kWaves * (kWave / (D / 8));
  const dim3 grid(p.n_split, p.n_kv_heads, p.batch);
  if (code == PRCR_E4M3)
    quant_decode_kernel<D, GT, kPaged, true><<<grid, kWaves * kWave, 0, stream>>>(p);
  else
    quant_decode_kernel<D, GT, kPaged, false><<<grid, kWaves * kWave, 0, stream>>>(p);
}

template <int D, int GT>
void launch_layout(const QuantDecodeParams &p, prcr_code code, bool paged, hipStream_t stream) {
  if (paged)
    launch_one<D, GT, true>(p, code, stream);
  else
    launch_one<D, GT, false>(p, code, stream);
}

}  // namespace

hipError_t launch_quant_decode(const QuantDecodeParams &in, prcr_code code, int head_dim, bool paged, hipStream_t stream) {
  QuantDecodeParams p = in;
  p.group = p.n_q_heads / p.n_kv_heads;
  p.waves = kWaves;
  p.fill = p.n_split;
  p.min_keys = 0;
  p.round = kWaves * (kWave / (head_dim / 8));
  auto inverse = [](int64_t n) { return n > 1 ? static_cast<uint32_t>(((int64_t{1} << 32) + n - 1) / n) : 0u; };
  p.split_inverse = inverse(p.n_split);
  p.fill_inverse = inverse(p.fill);
  p.direct = p.n_split == 1;
  if (head_dim == 64)
    p.group <= 4 ? launch_layout<64, 4>(p, code, paged, stream) : launch_layout<64, 8>(p, code, paged, stream);
  else
    p.group <= 4 ? launch_layout<128, 4>(p, code, paged, stream) : launch_layout<128, 8>(p, code, paged, stream);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.direct ? e : launch_decode_merge(p, head_dim, paged, stream);
}

}  // namespace prcr
