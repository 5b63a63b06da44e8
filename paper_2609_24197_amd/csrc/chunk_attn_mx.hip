// Attention of a ragged chunk of new tokens over the 4-bit paged cache (mx.h).  Up to 128 rows of a request: chunk_few.h.  Past
// that, the units, queue and merge of the other caches (chunk_tile.h), with K and V widened to the type of q on their way
// into LDS: three prompts of about 6000 tokens, 32 and 8 heads of 128, take 1383 to 1474 us by the card (981 to 921 TFLOP/s),
// over a bf16 cache 1286.  The new tokens' own K and V are in the cache, or beside it as they are, where their keys follow the
// cached ones.
#include "chunk_few.h"
#include "chunk_tile.h"

namespace hspec {
namespace {

template <int D>
hipError_t launch_few_rows(const ChunkAttnArgs& a, hipStream_t s) {
  const MxTile t = mx_tile(a);
  if (t.rw == 1) return t.rows == 16 ? launch_few<Few<bf16, D, 1, 1>>(a, s) : launch_few<Few<bf16, D, 2, 1>>(a, s);
  return t.rw == 2 ? launch_few<Share<D, 2, 2>>(a, s) : launch_few<Share<D, 4, 1>>(a, s);
}
template <class T, int D>
hipError_t launch_tiles(const ChunkAttnArgs& a, hipStream_t s) {   // of chunk_bounds, past 128 rows
  return launch_units<Chunk<T, D, 4, chunk_key_tile(4, sizeof(T) == 4), false, true>>(a, s);
}

}  // namespace

hipError_t launch_few_f32(const ChunkAttnArgs& a, hipStream_t s);

hipError_t launch_chunk_attn_mx(const ChunkAttnArgs& a, hipStream_t s) {
  if (!a.columns || a.first) {
    hipLaunchKernelGGL(chunk_plan, dim3(1), dim3(PL_THREADS), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (a.columns) return a.f32 ? launch_few_f32(a, s) : a.D == 128 ? launch_few_rows<128>(a, s) : launch_few_rows<64>(a, s);
  if (a.f32) return a.D == 128 ? launch_tiles<float, 128>(a, s) : launch_tiles<float, 64>(a, s);
  return a.D == 128 ? launch_tiles<bf16, 128>(a, s) : launch_tiles<bf16, 64>(a, s);
}

}  // namespace hspec
