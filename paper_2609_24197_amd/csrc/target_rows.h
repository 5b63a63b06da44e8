// Which rows of a ragged batch belong to which request, checked: shared by the kernels that take one.
#pragma once
#include "common.h"
#include "target.h"

namespace hspec {

// Rows of request b: cu[b] .. cu[b+1] inside [0, T) and at most max_n of them, whatever cu holds.
struct ChunkRows {
  int row0, n;
  bool ok;
};
__device__ __forceinline__ ChunkRows chunk_rows(const int32_t* cu, int b, int T, int max_n) {
  const int s = cu[b], e = cu[b + 1];
  ChunkRows r;
  r.ok = s >= 0 && s <= e && e <= T && e - s <= max_n && (b > 0 || s == 0);
  r.row0 = min(max(s, 0), T);
  const int top = (int)min((long long)T, (long long)r.row0 + max_n);
  r.n = min(max(e, r.row0), top) - r.row0;
  return r;
}

// Cached length of a request that takes n new tokens, in a cache that holds cap positions.
struct ChunkPos {
  int L;
  bool ok;
};
__device__ __forceinline__ ChunkPos chunk_pos(int L, int n, int cap) {
  ChunkPos p;
  const int top = max(cap - n, 0);
  p.ok = L >= 0 && n <= cap && L <= top;
  p.L = min(max(L, 0), top);
  return p;
}

// Request whose rows hold row r (the last b with cu[b] <= r), or -1 past the last one.  Every lane of a wave
// calls it; each round looks at 64 evenly spaced entries, so 64 requests take one load and 32767 three.
__device__ __forceinline__ int row_request(const int32_t* cu, int B, int r) {
  const int lane = threadIdx.x & 63;
  if (r >= cu[B]) return -1;
  int lo = 0, n = B;                       // the answer is in [lo, lo + n), if cu increases
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = lo + lane * step;
    const bool below = lane * step < n && cu[at] <= r;
    const int hits = max(__popcll(__ballot(below)), 1);
    const int from = lo + (hits - 1) * step;
    n = min(step, lo + n - from);
    lo = from;
  }
  return lo;
}

}  // namespace hspec
