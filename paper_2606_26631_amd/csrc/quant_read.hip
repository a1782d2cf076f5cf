// Reading one layer of the decoder cache in 8 bits back into rows of the model's type: what
// operators on several tokens, which take a cache of that type, need.  A row's codes times its
// scale, in float32, rounded once to that type.
#include "quant.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t bf16_nearest(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? 0x7FC0u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// A workgroup takes kSlots slots of one sequence and head; a thread 16 bytes of an output row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(const QuantReadParams p) {
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  constexpr int kLanes = D / E;
  constexpr int kSlots = kThreads / kLanes;
  const uint32_t seq_head = p.by_chunk.divide(blockIdx.x);
  const int chunk = static_cast<int>(blockIdx.x - seq_head * static_cast<uint32_t>((p.s_out + kSlots - 1) / kSlots));
  const int b = static_cast<int>(p.by_heads.divide(seq_head)), h = static_cast<int>(seq_head) - b * p.from.n_kv_heads;
  const int len_in = p.cache_len[b], most = min(p.capacity, p.s_out), len = min(max(len_in, 0), most);
  if (len != len_in && chunk == 0 && h == 0 && threadIdx.x == 0 && p.err != nullptr) atomicOr(p.err, PRCR_DERR_CAPACITY);
  const int slot = chunk * kSlots + static_cast<int>(threadIdx.x) / kLanes, c = threadIdx.x % kLanes;
  if (slot >= len) return;
  const Place at = place_of(p.from, b, slot);
  if (at.flag != 0) {
    if (c == 0 && p.err != nullptr) atomicOr(p.err, at.flag);
    return;
  }
  const int64_t row = at.row + p.layer * p.from.layer_rows + static_cast<int64_t>(h) * p.from.head_rows;
  const int64_t scale_at = at.scale + p.layer * p.from.layer_scales + static_cast<int64_t>(h) * p.from.head_scales;
  const int64_t out = (static_cast<int64_t>(seq_head) * p.s_out + slot) * D + c * E;
  auto half = [&](const void *codes, const float *scales, void *to) {
    const float scale = scales[scale_at];
    const uint32_t *const in = reinterpret_cast<const uint32_t *>(static_cast<const char *>(codes) + row * D + c * E);
    float x[E];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) decode4(in[i], p.from.code == PRCR_E4M3, x + 4 * i);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = sizeof(T) == 4 ? __float_as_uint(x[i] * scale)
                            : bf16_nearest(x[2 * i % E] * scale) | bf16_nearest(x[(2 * i + 1) % E] * scale) << 16;
    store_nt(static_cast<T *>(to) + out, w);
  };
  half(p.from.k, p.from.k_scale, p.k);
  half(p.from.v, p.from.v_scale, p.v);
}

template <typename T, int D>
hipError_t launch(const QuantReadParams &in, hipStream_t stream) {
  QuantReadParams p = in;
  constexpr int kSlots = kThreads / (D * static_cast<int>(sizeof(T)) / 16);
  const int64_t chunks = (static_cast<int64_t>(p.s_out) + kSlots - 1) / kSlots;
  const int64_t blocks = chunks * p.batch * p.from.n_kv_heads;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  p.by_chunk = Divisor::of(static_cast<int32_t>(chunks));
  p.by_heads = Divisor::of(p.from.n_kv_heads);
  quant_read_kernel<T, D><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quant_read(const QuantReadParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  if (dtype == PRCR_F32) return head_dim == 64 ? launch<float, 64>(p, stream) : launch<float, 128>(p, stream);
  return head_dim == 64 ? launch<uint16_t, 64>(p, stream) : launch<uint16_t, 128>(p, stream);
}

}  // namespace prcr
