// The kernels over the 4-bit cache whose waves meet at bare barriers, for a look at their assembly.
#include "chunk_few.h"
#include "chunk_tile.h"

namespace hspec {
namespace {

template __global__ void few_kernel<Share<64, 2, 2>>(ChunkAttnArgs);
template __global__ void few_kernel<Share<64, 4, 1>>(ChunkAttnArgs);
template __global__ void few_redo_kernel<Share<64, 2, 2>>(ChunkAttnArgs);
template __global__ void few_redo_kernel<Share<64, 4, 1>>(ChunkAttnArgs);
template __global__ void chunk_attn_kernel<Chunk<bf16, 64, 4, 64, false, true>>(ChunkAttnArgs);
template __global__ void chunk_redo_kernel<Chunk<bf16, 64, 4, 64, false, true>>(ChunkAttnArgs);
template __global__ void chunk_attn_kernel<Chunk<float, 64, 4, 32, false, true>>(ChunkAttnArgs);

}  // namespace
}  // namespace hspec
