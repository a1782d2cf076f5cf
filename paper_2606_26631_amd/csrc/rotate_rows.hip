// Rotation of query rows, before chunk attention and before the keys' weights: every row is
// turned at its own (t, h, w) position in double precision and rounded once to the stored
// type, as prefill capture rotates the keys.  The matrix products take operands of the
// stored type, so a query is rounded to it at some point; rounded here, the scores are
// those of two rows of the same kind, and their sums stay in float32.
//
// A workgroup takes kTokens tokens: their angles' cosines and sines once, into LDS, then
// all heads, 16 bytes of each half row per thread.  What bounds it is reading and writing
// the rows.  The first workgroup also reports what is wrong with the offsets and lengths,
// which the kernels after it only skip.
#include "attend.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kTokens = 8;
constexpr int kThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const AttendParams p) {
  constexpr int P = D / 2;
  constexpr int kPer = Store<T>::kPerChunk;
  constexpr int kChunks = P / kPer;          // of a half row
  __shared__ double s_cos[kTokens][P], s_sin[kTokens][P];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
  const int n = static_cast<int>(min(static_cast<int64_t>(kTokens), p.total_q - t0));
  if (blockIdx.x == 0 && p.err != nullptr) {
    int bits = 0;
    for (int b = threadIdx.x; b < p.batch; b += kThreads) {
      if (rows_of(p, b).bad || (b == 0 && p.q_off[0] < 0)) bits |= PRCR_DERR_OFFSETS;
      const int32_t len = p.cache_len[b];
      if (len != clamp_length(len, p.capacity)) bits |= PRCR_DERR_CAPACITY;
    }
    if (bits != 0) atomicOr(p.err, bits);
  }
  for (int i = threadIdx.x; i < n * P; i += kThreads) {
    const int t = i / P, pair = i % P;
    const double pos = static_cast<double>(p.q_pos[(t0 + t) * 3 + p.axis[pair]]);
    double sn, cs;
    sincos(pos * p.inv_freq[pair], &sn, &cs);
    s_cos[t][pair] = p.negate ? -cs : cs;
    s_sin[t][pair] = p.negate ? -sn : sn;
  }
  __syncthreads();
  const int per_token = p.n_q_heads * kChunks;
  for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
    const int t = i / per_token, c = i % kChunks;
    const int head = i % per_token / kChunks;
    const int64_t at = ((t0 + t) * p.n_q_heads + head) * (D * static_cast<int>(sizeof(T))) + c * 16;
    constexpr int kHalf = P * static_cast<int>(sizeof(T));
    const char *in = static_cast<const char *>(p.q) + at;
    char *out = static_cast<char *>(p.rotated) + at;
    u32x4 lo, hi;
    Store<T>::rotate(load_nt(in), load_nt(in + kHalf), &s_cos[t][c * kPer], &s_sin[t][c * kPer], lo, hi);
    *reinterpret_cast<u32x4 *>(out) = lo;
    *reinterpret_cast<u32x4 *>(out + kHalf) = hi;
  }
}

template <typename T>
hipError_t rotate(const AttendParams &p, int head_dim, hipStream_t stream) {
  const int64_t blocks = (static_cast<int64_t>(p.total_q) + kTokens - 1) / kTokens;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  if (head_dim == 64)
    rotate_rows_kernel<T, 64><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  else
    rotate_rows_kernel<T, 128><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const AttendParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  return dtype == PRCR_F32 ? rotate<float>(p, head_dim, stream) : rotate<uint16_t>(p, head_dim, stream);
}

}  // namespace prcr
