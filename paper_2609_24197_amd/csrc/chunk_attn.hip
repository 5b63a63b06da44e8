// Causal attention of a ragged chunk of new tokens over the paged cache that already holds them.
//
//   o[r, h] = sum_s p_s V[s],  p = softmax over visible s of scale q[r, h] . K[s],
//   visible: max(0, pos - window + 1) <= s <= pos = ctx_len + (r - first row of the request)
//
// A workgroup takes one KV head and a tile of 32 NW (token, query head of the group) rows of one request, and
// walks a range of the request's keys.  A wave owns 32 of those rows as the columns of
//   S^T [keys x rows] = K Q^T   and   O^T [D x rows] += V^T P^T,
// 32 x 32 products: S^T leaves a lane with 16 keys of one row per 32-key block, so the running maximum needs one
// exchange between the wave's halves per tile, the running sum none until the end, and P^T is already in the
// layout of the second product's operand if V^T is read with its keys in the same order (they are summed over, so
// any order serves).  K and V tiles stream into LDS by direct DMA, the next tile while one is multiplied; in a page
// a wave's 16 rows are consecutive, so a tile costs a wave one page id.
//
// Kernels: the plan (one workgroup: checks, list of units with the longest first, clears), the units, those of
// them with values that are not finite once more where requests can have several new tokens, and the merge of rows
// whose keys were split.  Few rows and long caches are split over keys so that the chip is full;
// pieces are merged in key order, so results do not depend on timing.
//
// fp32 storage takes the fp32 matrix products (32 x 32 x 2), so nothing is rounded below 32 bits.
//
// Bound by reading K and V where requests have few rows (64 requests x 1 token, 512..8192 cached, 32 and 8 heads of
// 128: 212 us for 1.2 GB; x 17 tokens 255), by the matrix and vector units in prompts, busy in 52 % and 46 % of the
// cycles and mostly in turn (three of about 6000 tokens 1278 us, 1064 TFLOP/s; 2000 tokens behind 30000, 64 heads,
// 1834 us, 1107; cards differ by up to 6 %; where a rule below has two figures, both are of one card).
#include "chunk_tile.h"

namespace hspec {
namespace {

// The instance of a tile (chunk_bounds).
template <class F>
auto with_variant(const ChunkAttnArgs& a, F f) {
  auto by_rows = [&](auto t, auto d) {
    typedef typename decltype(t)::type T;
    constexpr int D = decltype(d)::value;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int KT4 = chunk_key_tile(4, F32);
    if (a.tile_rows == 32) return f(Chunk<T, D, 1, chunk_key_tile(1, F32), true>{});
    if constexpr (F32)
      if (a.tile_rows == 64) return f(Chunk<T, D, 2, chunk_key_tile(2, F32), true>{});
    return a.once ? f(Chunk<T, D, 4, KT4, true>{}) : f(Chunk<T, D, 4, KT4, false>{});
  };
  if (a.f32) return a.D == 128 ? by_rows(std::common_type<float>{}, Int<128>{}) : by_rows(std::common_type<float>{}, Int<64>{});
  return a.D == 128 ? by_rows(std::common_type<bf16>{}, Int<128>{}) : by_rows(std::common_type<bf16>{}, Int<64>{});
}

}  // namespace

hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(chunk_plan, dim3(1), dim3(PL_THREADS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  return with_variant(a, [&](auto c) { return launch_units<decltype(c)>(a, s); });
}

}  // namespace hspec
