// The plan in columns (chunk_plan.h) of up to 64 requests, found by every wave for itself, a request a lane: a kernel that
// has it in its own first steps needs no plan's launch ahead of it.  Nothing in it is particular to this chip's
// instructions, so that a test can run it on the host.
#pragma once
#include "chunk_plan.h"

namespace hspec {
namespace {

constexpr int CO_REQUESTS = 64;

// A lane's request: its rows and keys, its steps and those before it, its units and those before them (a unit's slot is its
// number); of the whole call the steps of a column and the status bits found.
struct LanePlan {
  int row0, n, L, k0, len, unit, pieces, bits;
  unsigned step, steps, S;
};
__device__ __forceinline__ unsigned lanes_before(unsigned v, unsigned& total) {   // sum over the lanes before this one, and over all
  unsigned sum = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned w = __shfl_up(sum, o);
    if ((int)(threadIdx.x & 63) >= o) sum += w;
  }
  total = __shfl(sum, 63);
  return sum - v;
}
__device__ __forceinline__ LanePlan lane_plan(const ChunkAttnArgs& a) {
  const int b = threadIdx.x & 63, g = a.Hq / a.Hkv;
  LanePlan p{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1};
  const int from = b < a.B ? a.cu[b] : 0, to = b < a.B ? a.cu[b + 1] : 0, held = b < a.B ? a.ctx_lens[b] : 0;
  int start = from, bits = 0;
  for (bool again = false;; again = true) {
    if (b < a.B) {
      ChunkRows r = clamp_rows(start, max(to, start), a.T, a.max_new);
      r.ok = r.ok && start == from && to >= from && (b > 0 || from == 0);
      const ChunkPos at = chunk_pos(held, r.n, a.cap, a.held);
      bits |= (r.ok ? 0 : ST_BAD_ROWS) | (at.ok ? 0 : ST_BAD_CTX_LEN);
      p.row0 = r.row0;
      p.n = r.n;
      p.L = at.L;
    }
    if (again || !__ballot((bits & ST_BAD_ROWS) != 0)) break;   // (uniform)
    // bad rows: those of each request begin behind all before it, so that no row is in two (see chunk_plan)
    int top = b < a.B ? max(from, 0) : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(top, o);
      if (b >= o) top = max(top, w);
    }
    start = top;
  }
  p.bits = (__ballot((bits & ST_BAD_ROWS) != 0) ? ST_BAD_ROWS : 0) | (__ballot((bits & ST_BAD_CTX_LEN) != 0) ? ST_BAD_CTX_LEN : 0);
  if (p.n > 0) {
    const TileKeys t = tile_keys(a, g, 0, p.n, p.L);
    p.k0 = t.k0;
    p.len = max(t.k1 - t.k0, 0);
    p.steps = max((p.len + a.key_tile - 1) / a.key_tile, 1);
  }
  unsigned all, units;   // (64 requests of fewer than 2^31 positions: fewer than 2^31 steps)
  p.step = lanes_before(p.steps, all);
  p.S = max((all + (unsigned)a.columns - 1) / (unsigned)a.columns, 1u);
  if (p.n > 0) p.pieces = (int)((p.step + p.steps - 1) / p.S - p.step / p.S) + 1;
  p.unit = (int)lanes_before((unsigned)p.pieces, units);
  return p;
}
// What column w has in common with the lane's request: written to out[..] by its lane, in the order of the requests.
// Returns how many there are.
__device__ __forceinline__ int column_units(const ChunkAttnArgs& a, const LanePlan& p, int w, ChunkUnit* out) {
  const int b = threadIdx.x & 63;
  const unsigned long long s0 = (unsigned long long)w * p.S, s1 = s0 + p.S;
  const bool in = p.n > 0 && p.step < s1 && (unsigned long long)p.step + p.steps > s0;
  const unsigned long long mask = __ballot(in);
  if (in && out) {
    const long long at0 = s0 > p.step ? (long long)(s0 - p.step) * a.key_tile : 0;
    const long long at1 = min((long long)p.len, (long long)(s1 - p.step) * a.key_tile);
    out[__popcll(mask & ((1ULL << b) - 1))] =
        ChunkUnit{b, 0, p.k0 + (int)at0, p.k0 + (int)at1, p.pieces > 1 ? p.unit + w - (int)(p.step / p.S) : -1, p.row0, p.n, p.L};
  }
  return __popcll(mask);
}
// What the kernels behind need of the whole call, by one wave: the split tiles (an entry a request, fewer than two pieces:
// none), the status.
__device__ __forceinline__ void write_plan(const ChunkAttnArgs& a, const LanePlan& p) {
  const int b = threadIdx.x & 63;
  if (b < a.B) a.splits[b] = ChunkSplit{b, 0, p.unit, p.pieces, p.row0, p.n, p.L, 0};
  if (b == 0) {
    a.status[0] = p.bits;
    a.status[2] = a.B;
  }
}

}  // namespace
}  // namespace hspec
