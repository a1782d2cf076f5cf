// Rotation of query rows, before chunk attention and before the keys' weights: every row is
// turned at its own (t, h, w) position in double precision and rounded once to the stored
// type, as prefill capture rotates the keys.  The matrix products take operands of the
// stored type, so a query is rounded to it at some point; rounded here, the scores are
// those of two rows of the same kind, and their sums stay in float32.
//
// A thread takes 16 bytes of each half of a token's rows: their angles' cosines and sines
// once, then the rows of up to kHeads heads, all read before the first is turned.  What
// bounds it is reading and writing the rows.  The first workgroup also reports what is wrong
// with the offsets and lengths, which the kernels after it only skip.
#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kHeads = 8;
constexpr int kThreads = 64;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const AttendParams p, const Divisor by_groups,
                                                               const int n_groups, const int64_t n) {
  constexpr int P = D / 2;
  constexpr int kPer = Store<T>::kPerChunk;
  constexpr int kChunks = P / kPer;          // of a half row
  constexpr int kRowBytes = D * static_cast<int>(sizeof(T)), kHalf = kRowBytes / 2;
  if (blockIdx.x == 0 && p.err != nullptr) {
    int bits = 0;
    for (int b = threadIdx.x; b < p.batch; b += kThreads) {
      if (rows_of(p, b).bad) bits |= PRCR_DERR_OFFSETS;
      const int32_t len = p.cache_len[b];
      if (len != clamp_length(len, p.capacity)) bits |= PRCR_DERR_CAPACITY;
    }
    if (bits != 0) atomicOr(p.err, bits);
  }
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (id >= n) return;
  const int c = static_cast<int>(id % kChunks);
  const uint32_t unit = static_cast<uint32_t>(id / kChunks);        // token and group of heads (below 2^31)
  const uint32_t t = by_groups.divide(unit);
  const int h0 = static_cast<int>(unit - t * static_cast<uint32_t>(n_groups)) * kHeads;
  const int64_t at = (static_cast<int64_t>(t) * p.n_q_heads + h0) * kRowBytes + c * 16;
  const char *const in = static_cast<const char *>(p.q) + at;
  char *const out = static_cast<char *>(p.rotated) + at;
  const int heads = min(kHeads, p.n_q_heads - h0);
  u32x4 lo[kHeads], hi[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const char *const row = in + min(h, heads - 1) * kRowBytes;
    lo[h] = load_nt(row);
    hi[h] = load_nt(row + kHalf);
  }
  double cs[kPer], sn[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int pair = c * kPer + e;
    sincos(static_cast<double>(p.q_pos[static_cast<int64_t>(t) * 3 + p.axis[pair]]) * p.inv_freq[pair], &sn[e], &cs[e]);
    if (p.negate) {
      cs[e] = -cs[e];
      sn[e] = -sn[e];
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h >= heads) break;
    u32x4 a, b;
    Store<T>::rotate(lo[h], hi[h], cs, sn, a, b);
    *reinterpret_cast<u32x4 *>(out + h * kRowBytes) = a;
    *reinterpret_cast<u32x4 *>(out + h * kRowBytes + kHalf) = b;
  }
}

template <typename T, int D>
hipError_t rotate(const AttendParams &p, hipStream_t stream) {
  const int n_groups = (p.n_q_heads + kHeads - 1) / kHeads;
  const int64_t n = static_cast<int64_t>(p.total_q) * n_groups * (D / 2 / Store<T>::kPerChunk);
  const int64_t blocks = (n + kThreads - 1) / kThreads;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  rotate_rows_kernel<T, D><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p, Divisor::of(n_groups), n_groups, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const AttendParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  if (dtype == PRCR_F32) return head_dim == 64 ? rotate<float, 64>(p, stream) : rotate<float, 128>(p, stream);
  return head_dim == 64 ? rotate<uint16_t, 64>(p, stream) : rotate<uint16_t, 128>(p, stream);
}

}  // namespace prcr
