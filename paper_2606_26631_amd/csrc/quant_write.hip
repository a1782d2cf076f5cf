// Writing the decoder cache in 8 bits: tokens' keys and values as a layer makes them (append),
// and revisited visual tokens from the memory in every layer (rebind).  A key row is turned at
// the token's position, as a cache of the rows' type holds it, and then it and the value row
// are quantised: their largest magnitude, the scale, the codes.
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

// A lane's elements of a row, E of each half, as float32, and their largest magnitude's bits.
template <typename T>
__device__ __forceinline__ uint32_t elements(u32x4 lo, u32x4 hi, float *x) {
  uint32_t most = 0u;
  constexpr int E = Store<T>::kPerChunk;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 2) {
      x[2 * q] = __uint_as_float(lo[q] << 16);
      x[2 * q + 1] = __uint_as_float(lo[q] & 0xFFFF0000u);
      x[E + 2 * q] = __uint_as_float(hi[q] << 16);
      x[E + 2 * q + 1] = __uint_as_float(hi[q] & 0xFFFF0000u);
    } else {
      x[q] = __uint_as_float(lo[q]);
      x[E + q] = __uint_as_float(hi[q]);
    }
  }
#pragma unroll
  for (int e = 0; e < 2 * E; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  return most;
}

// Four codes in a word.
__device__ __forceinline__ uint32_t encode4(const float *x, float inverse, bool e4m3) {
  if (e4m3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inverse, x[1] * inverse, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inverse, x[3] * inverse, w, true));
  }
  uint32_t w = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    // (at least one product and sum each rounded by itself: no fused multiply-add)
    const float y = __fmul_rn(x[e], inverse);
    w |= (static_cast<uint32_t>(static_cast<int>(rintf(y))) & 0xFFu) << (8 * e);
  }
  return w;
}

template <typename T, int D, bool kRebind>
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
    if (blockIdx.x == 0 && blockIdx.y == 0)
      for (int b = threadIdx.x; b < p.batch; b += kWaves * kWave) {
        const int s0 = p.sel_off[b], s1 = p.sel_off[b + 1];
        if (p.new_len != nullptr) p.new_len[b] = p.start[b] + (s1 - s0);
        const bool bad = s1 < s0 || (b == 0 && s0 != 0) || (b == p.batch - 1 && s1 != p.n_tok);
        if (bad && p.err != nullptr) atomicOr(p.err, PRCR_DERR_OFFSETS);
      }
  }
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int c = lane % kLanes;
  const int64_t t64 = (static_cast<int64_t>(blockIdx.x) * kWaves + wave) * kTokens + lane / kLanes;
  if (t64 >= p.n_tok) return;
  const int t = static_cast<int>(t64);
  const int row0 = static_cast<int>(blockIdx.y) * p.rows_per_wave, row1 = min(row0 + p.rows_per_wave, p.rows);
  const bool tells = c == 0 && blockIdx.y == 0;   // the lane that reports for its token

  // The token: its sequence, position, slot, and where its rows come from.
  int b, flag = 0;
  double pos[3];
  int64_t slot, source;                      // source: index of the token's first row
  int64_t v_from = -1, v_from_scale = 0;     // of a memory without values: the slot's bases
  if constexpr (kRebind) {
    int lo = 0, hi = p.batch;                // the last sequence that begins at or before t
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (mid <= p.batch && p.sel_off[mid] <= t) lo = mid; else hi = mid - 1;
    }
    b = min(lo, p.batch - 1);
    const int s0 = p.sel_off[b], s1 = p.sel_off[b + 1], m = p.sel_idx[t];
    const bool offsets_ok = lo < p.batch && s0 >= 0 && s0 <= t && t < s1 && s1 <= p.n_tok;
    const int64_t len = p.start[b];
    slot = len + (t - s0);
    if (!offsets_ok)
      flag = PRCR_DERR_OFFSETS;
    else if (m < 0 || m >= p.n_visual[b] || m >= p.max_visual)
      flag = PRCR_DERR_INDEX;
    else if (p.v_slot != nullptr) {
      const int64_t vs = p.v_slot[static_cast<int64_t>(b) * p.max_visual + m];
      if (vs < 0 || vs >= len) {
        flag = PRCR_DERR_INDEX;
      } else {
        const Place from = place_of(to, b, vs);
        flag = from.flag;
        v_from = from.row;
        v_from_scale = from.scale;
      }
    }
    source = (static_cast<int64_t>(b) * p.max_visual + m) * p.rows;
#pragma unroll
    for (int a = 0; a < 3; ++a) pos[a] = p.new_pos[3 * static_cast<int64_t>(t) + a];
  } else {
    b = static_cast<int>(p.by_seq.divide(static_cast<uint32_t>(t)));
    const int s = t - b * p.s_src, n = p.n_tokens[b];
    if ((n < 0 || n > p.s_src) && s == 0 && tells && p.err != nullptr) atomicOr(p.err, PRCR_DERR_INDEX);
    if (s >= n) return;
    slot = static_cast<int64_t>(p.start[b]) + s;
    source = static_cast<int64_t>(t) * H;
#pragma unroll
    for (int a = 0; a < 3; ++a) pos[a] = p.pos[3 * static_cast<int64_t>(t) + a];
  }
  Place at{0, 0, -1, 0};
  if (flag == 0) {
    at = place_of(to, b, slot);
    flag = at.flag;
  }
  if (tells) {
    if (flag != 0 && p.err != nullptr) atomicOr(p.err, flag);
    if (kRebind && p.slot_mapping != nullptr) p.slot_mapping[t] = flag == 0 ? at.id : -1;
  }
  if (flag != 0) return;

  double cs[E], sn[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = c * E + e, ax = p.axis[i];
    turn((ax == 0 ? pos[0] : ax == 1 ? pos[1] : pos[2]) * p.inv_freq[i], &sn[e], &cs[e]);
  }

  // Quantises a row and stores it: 2 E codes a lane (E of each half, brought together with the
  // neighbour's), and the scale.
  auto put = [&](u32x4 lo, u32x4 hi, void *codes, float *scales, int64_t row, int64_t scale_at) {
    float x[2 * E];
    const uint32_t most = group_max<kLanes>(elements<T>(lo, hi, x));
    const bool finite = most < 0x7F800000u, e4m3 = to.code == PRCR_E4M3;
    const float scale = finite ? fmaxf(__uint_as_float(most) / (e4m3 ? 448.f : 127.f), FLT_MIN) : __uint_as_float(0x7FC00000u);
    const float inverse = 1.f / scale;
    uint32_t w[2 * E / 4];
#pragma unroll
    for (int i = 0; i < 2 * E / 4; ++i) w[i] = finite ? encode4(x + 4 * i, inverse, e4m3) : 0u;
    char *const at = static_cast<char *>(codes) + row * D;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      *reinterpret_cast<uint32_t *>(at + c * E + 4 * i) = w[i];
      *reinterpret_cast<uint32_t *>(at + P + c * E + 4 * i) = w[E / 4 + i];
    }
    if (c == 0) scales[scale_at] = scale;
  };
  for (int r = row0; r < row1; ++r) {
    const int l = kRebind ? static_cast<int>(p.by_heads.divide(static_cast<uint32_t>(r))) : p.layer;
    const int h = kRebind ? r - l * H : r;
    const int64_t row = at.row + l * to.layer_rows + static_cast<int64_t>(h) * to.head_rows;
    const int64_t scale_at = at.scale + l * to.layer_scales + static_cast<int64_t>(h) * to.head_scales;
    const int64_t from = (source + r) * kRowBytes + c * 16;
    const char *const k = static_cast<const char *>(p.k) + from;
    u32x4 lo = load_nt(k), hi = load_nt(k + kHalfBytes), ol, oh;
    Store<T>::rotate(lo, hi, cs, sn, ol, oh);
    put(ol, oh, to.k, to.k_scale, row, scale_at);
    if (kRebind && p.v_slot != nullptr) {
      const int64_t r2 = v_from + l * to.layer_rows + static_cast<int64_t>(h) * to.head_rows;
      const char *const in = static_cast<const char *>(to.v) + r2 * D;
      char *const out = static_cast<char *>(to.v) + row * D;
#pragma unroll
      for (int i = 0; i < 2 * E / 4; ++i)
        *reinterpret_cast<uint32_t *>(out + c * 2 * E + 4 * i) = *reinterpret_cast<const uint32_t *>(in + c * 2 * E + 4 * i);
      if (c == 0)
        to.v_scale[scale_at] = to.v_scale[v_from_scale + l * to.layer_scales + static_cast<int64_t>(h) * to.head_scales];
    } else {
      const char *const v = static_cast<const char *>(p.v) + from;
      lo = load_nt(v);
      hi = load_nt(v + kHalfBytes);
      put(lo, hi, to.v, to.v_scale, row, scale_at);
    }
  }
}

template <typename T, int D, bool kRebind>
hipError_t launch(const QuantWriteParams &in, hipStream_t stream) {
  QuantWriteParams p = in;
  constexpr int kTokens = kWave / (D / 2 / Store<T>::kPerChunk);
  p.by_seq = Divisor::of(kRebind ? 1 : p.s_src);
  p.by_heads = Divisor::of(p.to.n_kv_heads);
  p.rows_per_wave = 8;
  while ((p.rows + p.rows_per_wave - 1) / p.rows_per_wave > 65535) p.rows_per_wave *= 2;
  const int64_t blocks = std::max<int64_t>(1, (static_cast<int64_t>(p.n_tok) + kWaves * kTokens - 1) / (kWaves * kTokens));
  if (!grid_fits(blocks, kWaves * kWave)) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks), (p.rows + p.rows_per_wave - 1) / p.rows_per_wave);
  quant_write_kernel<T, D, kRebind><<<grid, kWaves * kWave, 0, stream>>>(p);
  return hipGetLastError();
}

template <bool kRebind>
hipError_t dispatch(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  if (dtype == PRCR_F32)
    return head_dim == 64 ? launch<float, 64, kRebind>(p, stream) : launch<float, 128, kRebind>(p, stream);
  return head_dim == 64 ? launch<uint16_t, 64, kRebind>(p, stream) : launch<uint16_t, 128, kRebind>(p, stream);
}

}  // namespace

hipError_t launch_quant_append(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dispatch<false>(p, dtype, head_dim, stream);
}
hipError_t launch_quant_rebind(const QuantWriteParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dispatch<true>(p, dtype, head_dim, stream);
}

}  // namespace prcr
