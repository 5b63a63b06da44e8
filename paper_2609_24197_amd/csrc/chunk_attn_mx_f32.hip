// The few rows of attention over the 4-bit cache (chunk_few.h) with fp32 rows.
#include "chunk_few.h"

namespace hspec {
namespace {

template <int D>
hipError_t launch_waves(const ChunkAttnArgs& a, hipStream_t s) {
  switch (mx_tile(a).rw) {
    case 1: return launch_few<Few<float, D, 1, 1>>(a, s);
    case 2: return launch_few<Few<float, D, 1, 2>>(a, s);
    case 4: return launch_few<Few<float, D, 1, 4>>(a, s);
    default: return launch_few<Few<float, D, 1, 8>>(a, s);
  }
}

}  // namespace

hipError_t launch_few_f32(const ChunkAttnArgs& a, hipStream_t s) {
  return a.D == 128 ? launch_waves<128>(a, s) : launch_waves<64>(a, s);
}

}  // namespace hspec
