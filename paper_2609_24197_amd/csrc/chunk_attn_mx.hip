// Attention of a ragged chunk of new tokens over the 4-bit paged cache (mx.h): the units, tiles and merge of the other
// caches' (chunk_tile.h), with K and V widened to the type of q on their way into LDS.  The new tokens' own K and V are
// in the cache, or beside it as they are, where their keys follow the cached ones.
#include "chunk_few.h"
#include "chunk_tile.h"

namespace hspec {
namespace {

template <class F>
auto with_variant(const ChunkAttnArgs& a, F f) {
  auto by_rows = [&](auto t, auto d) {
    typedef typename decltype(t)::type T;
    constexpr int D = decltype(d)::value;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int KT4 = chunk_key_tile(4, F32);
    if constexpr (F32) {   // (bf16 has more rows than that)
      if (a.tile_rows == 32) return f(Chunk<T, D, 1, chunk_key_tile(1, F32), true, true>{});
      if (a.tile_rows == 64) return f(Chunk<T, D, 2, chunk_key_tile(2, F32), true, true>{});
    }
    return a.once ? f(Chunk<T, D, 4, KT4, true, true>{}) : f(Chunk<T, D, 4, KT4, false, true>{});
  };
  if (a.f32) return a.D == 128 ? by_rows(std::common_type<float>{}, Int<128>{}) : by_rows(std::common_type<float>{}, Int<64>{});
  return a.D == 128 ? by_rows(std::common_type<bf16>{}, Int<128>{}) : by_rows(std::common_type<bf16>{}, Int<64>{});
}

template <int D>
hipError_t launch_few_rows(const ChunkAttnArgs& a, hipStream_t s) {
  const MxTile t = mx_tile(a);
  if (t.rw == 1) return t.ct == 1 ? launch_few<Few<D, 1>>(a, s) : launch_few<Few<D, 2>>(a, s);
  return t.rw == 2 ? launch_few<Share<D, 2, 2>>(a, s) : launch_few<Share<D, 4, 1>>(a, s);
}

}  // namespace

hipError_t launch_chunk_attn_mx(const ChunkAttnArgs& a, hipStream_t s) {
  if (!a.columns || a.first) {
    hipLaunchKernelGGL(chunk_plan, dim3(1), dim3(PL_THREADS), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (a.columns) return a.D == 128 ? launch_few_rows<128>(a, s) : launch_few_rows<64>(a, s);
  return with_variant(a, [&](auto c) { return launch_units<decltype(c)>(a, s); });
}

}  // namespace hspec
