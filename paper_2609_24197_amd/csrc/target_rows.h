// Which rows of a ragged batch belong to which request, checked: shared by the kernels that take one.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

namespace hspec {

// Rows of request b: cu[b] .. cu[b+1] inside [0, T) and at most max_n of them, whatever cu holds.
struct ChunkRows {
  int row0, n;
  bool ok;
};
__device__ __forceinline__ ChunkRows clamp_rows(int s, int e, int T, int max_n) {
  ChunkRows r;
  r.ok = s >= 0 && s <= e && e <= T && e - s <= max_n;
  r.row0 = min(max(s, 0), T);
  const int top = (int)min((long long)T, (long long)r.row0 + max_n);
  r.n = min(max(e, r.row0), top) - r.row0;
  return r;
}
__device__ __forceinline__ ChunkRows chunk_rows(const int32_t* cu, int b, int T, int max_n) {
  const int s = cu[b];
  ChunkRows r = clamp_rows(s, cu[b + 1], T, max_n);
  r.ok = r.ok && (b > 0 || s == 0);
  return r;
}

// Whether the range of request i, of those before request b, holds some of the n rows from r0 on: [from, to) of them.
struct RowsBefore {
  int from, to;
};
__device__ __forceinline__ RowsBefore rows_before(const int32_t* cu, int i, int b, int T, int max_n, int r0, int n) {
  RowsBefore r{0, 0};
  if (i < b) {
    const ChunkRows c = clamp_rows(cu[i], cu[i + 1], T, max_n);
    r.from = max(c.row0 - r0, 0);
    r.to = min(c.row0 + c.n - r0, n);
  }
  return r;
}
// Of the n <= 64 rows from r0 on of request b, those that are also of a request before it (where cu is bad): bit i for
// row r0 + i.  Every lane of a wave calls it.
__device__ __forceinline__ unsigned long long rows_taken(const int32_t* cu, int b, int T, int max_n, int r0, int n) {
  unsigned long long taken = 0;
  for (int at = 0; at < b; at += 64) {
    const RowsBefore r = rows_before(cu, at + (int)(threadIdx.x & 63), b, T, max_n, r0, n);
    for (unsigned long long left = __ballot(r.from < r.to); left; left &= left - 1) {
      const int lane = __builtin_ctzll(left), from = __shfl(r.from, lane), to = __shfl(r.to, lane);
      taken |= ~0ULL >> (64 - (to - from)) << from;
    }
  }
  return taken;
}

// Cached length of a request that takes n new tokens: at most cap positions in all, and `held` of them cached.
struct ChunkPos {
  int L;
  bool ok;
};
__device__ __forceinline__ ChunkPos chunk_pos(int L, int n, int cap, int held = INT_MAX) {
  ChunkPos p;
  const int top = min(max(cap - n, 0), held);
  p.ok = L >= 0 && n <= cap && L <= top;
  p.L = min(max(L, 0), top);
  return p;
}

// Where row r belongs: request b, token i of its n new ones, L cached before them; n = 0 for a row of no request.
// Every lane of a wave calls it.
struct RowPlace {
  int b, i, n, L;
};
__device__ __forceinline__ RowPlace row_place(const int32_t* cu, const int32_t* ctx_lens, int B, int T, int max_n, int r) {
  const int lane = threadIdx.x & 63;
  RowPlace p{0, 0, 0, 0};
  if (B <= 64) {   // one round trip for all of it: a lane holds each request's first row and length
    const int end = cu[B];
    const int first = cu[min(lane, B)], len = ctx_lens[min(lane, B - 1)];
    const int hits = __popcll(__ballot(lane < B && first <= r));
    if (hits == 0 || r >= min(end, T)) return p;
    p.b = hits - 1;
    p.L = __shfl(len, p.b);
    const int s = __shfl(first, p.b), e = hits < 64 ? __shfl(first, hits) : end;
    const ChunkRows c = clamp_rows(s, e, T, max_n);
    p.i = r - c.row0;
    p.n = p.i >= 0 && p.i < c.n ? c.n : 0;
    return p;
  }
  if (r >= min(cu[B], T)) return p;
  int lo = 0, n = B;   // the last b with cu[b] <= r is in [lo, lo + n), if cu increases; 64 evenly spaced entries a round
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = lo + lane * step;
    const bool below = lane * step < n && cu[at] <= r;
    const int hits = max(__popcll(__ballot(below)), 1);
    const int from = lo + (hits - 1) * step;
    n = min(step, lo + n - from);
    lo = from;
  }
  const ChunkRows c = chunk_rows(cu, lo, T, max_n);
  p.b = lo;
  p.L = ctx_lens[lo];
  p.i = r - c.row0;
  p.n = p.i >= 0 && p.i < c.n ? c.n : 0;
  return p;
}

}  // namespace hspec
