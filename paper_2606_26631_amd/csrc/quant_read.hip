// Reading one layer of the decoder cache in 8 bits back into rows of the model's type: what
// operators on several tokens, which take a cache of that type, need.  A row's codes times its
// scale, in float32, rounded once to that type.
//
// A thread takes 16 bytes of one slot's output rows, of its key and its value; a workgroup consecutive
// slots of a sequence and head.  What bounds it is reading the codes and writing the rows: 64 paged
// sequences of 2,912-6,512 slots, 4 heads, bf16, 919 MB in 158 us (5.8 TB/s).  Threads with more slots of
// their own, all read before the first is written, are slower: two 165, four 173, eight 180.  The
// rows are written past the caches (190 us with four slots a thread through them, 177 past them), the codes
// read through them: half lines of 64 features would be read twice past them (107 and 90 us, head_dim 64).
#include "attend.h"
#include "quant.h"
#include "rotary.h"

namespace prcr {
namespace {

constexpr int kThreads = 256;

template <typename T, int D>
struct Shape {
  static constexpr int kPer = 16 / static_cast<int>(sizeof(T));   // elements of a thread
  static constexpr int kLanes = D / kPer;                         // threads of a row
  static constexpr int kSlots = kThreads / kLanes;                // slots of a workgroup
};

template <typename T, int D, bool kE4M3>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(const QuantReadParams p) {
  typedef Shape<T, D> S;
  constexpr int kPer = S::kPer;
  typedef uint32_t code_words __attribute__((ext_vector_type(kPer / 4)));
  const QuantStore &from = p.from;
  const uint32_t chunks = (static_cast<uint32_t>(p.s_out) + S::kSlots - 1) / S::kSlots;
  const uint32_t seq_head = p.by_chunk.divide(blockIdx.x);
  const int chunk = static_cast<int>(blockIdx.x - seq_head * chunks);
  const int b = static_cast<int>(p.by_heads.divide(seq_head)), h = static_cast<int>(seq_head) - b * from.n_kv_heads;
  const int len_in = p.cache_len[b], most = min(p.capacity, p.s_out), len = min(max(len_in, 0), most);
  if (len != len_in && chunk == 0 && h == 0 && threadIdx.x == 0 && p.err != nullptr) atomicOr(p.err, PRCR_DERR_CAPACITY);
  const int slot = chunk * S::kSlots + static_cast<int>(threadIdx.x) / S::kLanes, c = threadIdx.x % S::kLanes;
  if (slot >= len) return;
  const Place at = place_of(from, b, entry_of_slot(from, b, slot));
  if (at.flag != 0) {
    if (c == 0 && p.err != nullptr) atomicOr(p.err, at.flag);
    return;
  }
  const int64_t row = at.row + p.layer * from.layer_rows + static_cast<int64_t>(h) * from.head_rows;
  const int64_t scale_at = at.scale + p.layer * from.layer_scales + static_cast<int64_t>(h) * from.head_scales;
  const int64_t in = row * D + c * kPer, out = (static_cast<int64_t>(seq_head) * p.s_out + slot) * D + c * kPer;
  const code_words k = *reinterpret_cast<const code_words *>(static_cast<const char *>(from.k) + in);
  const code_words v = *reinterpret_cast<const code_words *>(static_cast<const char *>(from.v) + in);
  const float k_scale = from.k_scale[scale_at], v_scale = from.v_scale[scale_at];
  auto put = [&](code_words w, float scale, void *rows) {
    float y[kPer];
#pragma unroll
    for (int j = 0; j < kPer / 4; ++j) decode4(w[j], kE4M3, y + 4 * j);
    u32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4)
        o[j] = __float_as_uint(y[j] * scale);
      else
        o[j] = pack_bf16(y[2 * j] * scale, y[2 * j + 1] * scale);
    }
    store_nt(static_cast<T *>(rows) + out, o);
  };
  put(k, k_scale, p.k);
  put(v, v_scale, p.v);
}

template <typename T, int D, bool kE4M3>
hipError_t launch(const QuantReadParams &in, hipStream_t stream) {
  QuantReadParams p = in;
  const int64_t chunks = (static_cast<int64_t>(p.s_out) + Shape<T, D>::kSlots - 1) / Shape<T, D>::kSlots;
  const int64_t blocks = chunks * p.batch * p.from.n_kv_heads;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  p.by_chunk = Divisor::of(static_cast<int32_t>(chunks));
  p.by_heads = Divisor::of(p.from.n_kv_heads);
  quant_read_kernel<T, D, kE4M3><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t dispatch_code(const QuantReadParams &p, hipStream_t stream) {
  return p.from.code == PRCR_E4M3 ? launch<T, D, true>(p, stream) : launch<T, D, false>(p, stream);
}

}  // namespace

hipError_t launch_quant_read(const QuantReadParams &p, prcr_dtype dtype, int head_dim, hipStream_t stream) {
  if (dtype == PRCR_F32) return head_dim == 64 ? dispatch_code<float, 64>(p, stream) : dispatch_code<float, 128>(p, stream);
  return head_dim == 64 ? dispatch_code<uint16_t, 64>(p, stream) : dispatch_code<uint16_t, 128>(p, stream);
}

}  // namespace prcr
