// Rotation of query rows, before the keys' weights are summed: every row that counts is
// turned at its own (t, h, w) position in double precision and rounded once to the stored
// type, as prefill capture rotates the keys (chunk attention, which reads a row only for
// its own tile, turns it there).  The matrix products take operands of the stored type, so
// a query is rounded to it at some point; rounded here, the scores are those of two rows of
// the same kind, and their sums stay in float32.
//
// A thread takes 16 bytes of each half of a token's rows: their angles' cosines and sines
// once, then the rows of kHeads heads, all read before the first is turned.  What bounds it
// is reading and writing the rows (10,240 tokens of 32 heads of 128, 168 MB: 32 us, 5.2 TB/s); of
// few rows, a thread's own work (32 tokens: 5.0 us).  The first workgroup also reports what
// is wrong with the offsets and lengths, which the kernels after it only skip.
#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kThreads = 64;

template <typename T, int D, int kHeads>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const AttendParams p, const Divisor by_groups,
                                                               const int n_groups, const int64_t n) {
  constexpr int P = D / 2;
  constexpr int kPer = Store<T>::kPerChunk;
  constexpr int kChunks = P / kPer;          // of a half row
  constexpr int kRowBytes = D * static_cast<int>(sizeof(T)), kHalf = kRowBytes / 2;
  if (blockIdx.x == 0 && p.err != nullptr) report(p, threadIdx.x, kThreads);
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (id >= n) return;
  const int c = static_cast<int>(id % kChunks);
  double freq[kPer];
  int axis[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    freq[e] = p.inv_freq[c * kPer + e];
    axis[e] = p.axis[c * kPer + e];
  }
  const uint32_t unit = static_cast<uint32_t>(id / kChunks);        // token and group of heads (below 2^31)
  const uint32_t token = by_groups.divide(unit);
  const int h0 = static_cast<int>(unit - token * static_cast<uint32_t>(n_groups)) * kHeads;
  uint32_t t = token;
  if (p.window > 0) {                        // the last `window` rows of each sequence
    const int b = static_cast<int>(p.by_split.divide(token)), i = static_cast<int>(token) - b * p.window;
    const Rows rows = rows_of(p, b);
    if (i >= rows.n) return;
    t = static_cast<uint32_t>(rows.start + rows.n - 1 - i);
  }
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
  int32_t pos[3];
#pragma unroll
  for (int a = 0; a < 3; ++a) pos[a] = p.q_pos[static_cast<int64_t>(t) * 3 + a];
  double cs[kPer], sn[kPer];
  f32x4 split[8];                            // (bf16: kPer is 8)
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int32_t at_axis = axis[e] == 0 ? pos[0] : axis[e] == 1 ? pos[1] : pos[2];
    turn(static_cast<double>(at_axis) * freq[e], &sn[e], &cs[e]);
    if (p.negate) {
      cs[e] = -cs[e];
      sn[e] = -sn[e];
    }
    if constexpr (sizeof(T) == 2) split[e] = split_angle(cs[e], sn[e]);
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h >= heads) break;
    u32x4 a = lo[h], b = hi[h];
    if constexpr (sizeof(T) == 2)
      turn_bf16(a, b, split);
    else
      Store<T>::rotate(lo[h], hi[h], cs, sn, a, b);
    *reinterpret_cast<u32x4 *>(out + h * kRowBytes) = a;
    *reinterpret_cast<u32x4 *>(out + h * kRowBytes + kHalf) = b;
  }
}

__global__ __launch_bounds__(kThreads) void report_kernel(const AttendParams p) { report(p, threadIdx.x, kThreads); }

template <typename T, int D, int kHeads>
hipError_t rotate(const AttendParams &in, hipStream_t stream) {
  AttendParams p = in;
  const int n_groups = (p.n_q_heads + kHeads - 1) / kHeads;
  // A window that covers more rows than there are is none.
  if (static_cast<int64_t>(p.window) * p.batch >= p.total_q) p.window = 0;
  if (p.window > 0) p.by_split = Divisor::of(p.window);
  const int64_t tokens = p.window > 0 ? static_cast<int64_t>(p.window) * p.batch : p.total_q;
  const int64_t n = tokens * n_groups * (D / 2 / Store<T>::kPerChunk);
  const int64_t blocks = (n + kThreads - 1) / kThreads;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  rotate_rows_kernel<T, D, kHeads><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p, Divisor::of(n_groups), n_groups, n);
  return hipGetLastError();
}

template <typename T>
hipError_t rotate_dim(const AttendParams &p, int head_dim, hipStream_t stream) {
  // bf16 rows in quantity: four heads a thread share the angles (2,560 tokens of 4 sequences: the
  // keys' weights take 185 us, with one 221); with a head a thread, fewer than 2^16 threads are less
  // than a wave on every SIMD (48 tokens: 10.4 us with one, 11.6 with four).  float32 rows, whose
  // turning is double precision throughout, gain nothing (the same 10,240 tokens: 1,056 and 1,058 us).
  if constexpr (sizeof(T) == 2)
    if (static_cast<int64_t>(p.total_q) * p.n_q_heads * (head_dim / 16) >= (1 << 16))
      return head_dim == 64 ? rotate<T, 64, 4>(p, stream) : rotate<T, 128, 4>(p, stream);
  return head_dim == 64 ? rotate<T, 64, 1>(p, stream) : rotate<T, 128, 1>(p, stream);
}

}  // namespace

hipError_t launch_report(const AttendParams &p, hipStream_t stream) {
  report_kernel<<<1, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_rotate(const AttendParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dtype == PRCR_F32 ? rotate_dim<float>(p, head_dim, stream) : rotate_dim<uint16_t>(p, head_dim, stream);
}

}  // namespace prcr
