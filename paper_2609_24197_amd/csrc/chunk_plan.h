// The plan of the chunk attention: checks of the call, list of its units, clears of its counters.  Nothing in it is
// particular to this chip's instructions, so that a test can run it on the host.
#pragma once
#include <hip/hip_runtime.h>

#include "status.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int PL_THREADS = 256;
constexpr int PL_BUCKETS = 64;

struct PlanLds {
  int first[PL_THREADS + 1];          // tiles before each request of the chunk
  int row0[PL_THREADS], n[PL_THREADS], L[PL_THREADS];
  int wave_sum[PL_THREADS / 64];
  int end;                            // the largest of cu before the chunk, where its rows are bad
  unsigned long long keys;            // keys of all tiles
  int longest, slots, n_splits, bits;
  int hist[PL_BUCKETS];
  // in columns: of each tile of the chunk its range of keys, the steps and the units before it, its first slot
  int k0[PL_THREADS], len[PL_THREADS], unit[PL_THREADS], slot[PL_THREADS];
  unsigned long long step[PL_THREADS], wave_steps[PL_THREADS / 64];
};

struct TileKeys {
  int k0, k1;   // key range, k0 a multiple of the key tile; k1 <= k0: no key
};
__device__ __forceinline__ TileKeys tile_keys(const ChunkAttnArgs& a, int g, int tile, int n, int L) {
  const int c0 = tile * a.tile_rows;
  const int t0 = c0 / g, t1 = (int)min((long long)c0 + a.tile_rows, (long long)n * g) - 1;
  TileKeys r;
  r.k1 = min(L + (a.block ? n : t1 / g + 1), a.cap);
  r.k0 = a.window > 0 ? max(L + t0 - a.window + 1, 0) / a.key_tile * a.key_tile : 0;
  return r;
}

// One workgroup lists the units.  Every tile of rows has len keys; tiles longer than S >= keys of all tiles x Hkv /
// target are cut into ceil(len / S) even pieces, so the pieces of all tiles number at most target / Hkv more than the
// tiles, and the split ones twice that (what the workspace holds).  Units are written longest first (64 classes of
// length), which keeps the queue's tail short.
//
// In columns (a.columns > 0, one tile a request): the steps of key_tile keys of all tiles, one tile behind the other, are
// cut into columns of the same number of steps, so that as many workgroups as run at once have the same to do; a unit is what a
// tile and a column have in common, and column w has units first[w] .. first[w + 1] - 1.
__global__ void __launch_bounds__(PL_THREADS) chunk_plan(ChunkAttnArgs a) {
  __shared__ PlanLds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = a.Hq / a.Hkv;
  if (tid < PL_BUCKETS) s.hist[tid] = 0;
  if (tid == 0) {
    s.keys = 0;
    s.longest = 0;
    s.slots = 0;
    s.n_splits = 0;
    s.bits = 0;
  }
  for (int i = tid; i < kChunkClasses * kChunkQueueStride; i += PL_THREADS) a.queue[i] = 0;

  // Requests [c0, c0 + PL_THREADS): rows, lengths and tile counts into LDS.  Returns the chunk's tiles.  Once a request's
  // rows are found bad, those of each begin behind all before it: no row is in two requests, so there are
  // never more tiles than the workspace holds.
  auto load = [&](int c0) -> int {
    __syncthreads();
    const int b = c0 + tid;
    const int from = b < a.B ? a.cu[b] : 0, to = b < a.B ? a.cu[b + 1] : 0, len = b < a.B ? a.ctx_lens[b] : 0;
    int start = from, before = 0, v = 0;
    for (bool again = false;; again = true) {
      int nt = 0;
      if (b < a.B) {
        ChunkRows r = clamp_rows(start, max(to, start), a.T, a.max_new);
        r.ok = r.ok && start == from && to >= from && (b > 0 || from == 0);
        const ChunkPos p = chunk_pos(len, r.n, a.cap, a.held);
        if (!r.ok || !p.ok) atomicOr(&s.bits, (r.ok ? 0 : ST_BAD_ROWS) | (p.ok ? 0 : ST_BAD_CTX_LEN));
        s.row0[tid] = r.row0;
        s.n[tid] = r.n;
        s.L[tid] = p.L;
        nt = (int)(((long long)r.n * g + a.tile_rows - 1) / a.tile_rows);
      }
      v = nt;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int w = __shfl_up(v, o);
        if (lane >= o) v += w;
      }
      if (lane == 63) s.wave_sum[wave] = v;
      if (tid == 0) s.end = 0;
      __syncthreads();
      before = 0;
      for (int w = 0; w < wave; ++w) before += s.wave_sum[w];
      if (again || !(s.bits & ST_BAD_ROWS)) break;   // (uniform)
      // the largest of cu up to this request
      int top = 0;
      for (int i = tid; i <= c0; i += PL_THREADS) top = max(top, a.cu[i]);
      atomicMax(&s.end, top);
      s.first[tid] = from;
      __syncthreads();
      start = s.end;
      for (int i = 0; i <= tid; ++i) start = max(start, s.first[i]);
      __syncthreads();
    }
    s.first[tid + 1] = before + v;
    if (tid == 0) s.first[0] = 0;
    __syncthreads();
    return s.first[PL_THREADS];
  };
  auto request_of = [&](int tile) -> int {   // of the chunk: the last with first <= tile
    int lo = 0;
#pragma unroll
    for (int st = PL_THREADS / 2; st > 0; st >>= 1)
      if (s.first[lo + st] <= tile) lo += st;
    return lo;
  };
  const int chunks = (a.B + PL_THREADS - 1) / PL_THREADS;
  int tiles = 0, all_tiles = 0;
  struct Tile {
    int r, tile, k0, len;
  };
  Tile mine{0, 0, 0, 0};   // this thread's first tile, where there is one chunk
  auto tile_of = [&](int t) -> Tile {
    const int r = request_of(t), tile = t - s.first[r];
    const TileKeys k = tile_keys(a, g, tile, s.n[r], s.L[r]);
    return Tile{r, tile, k.k0, max(k.k1 - k.k0, 0)};
  };
  auto each = [&](bool again, auto f) {
    for (int c = 0; c < chunks; ++c) {
      if (chunks > 1 || !again) tiles = load(c * PL_THREADS);
      if (!again) all_tiles += tiles;
      for (int t = tid; t < tiles; t += PL_THREADS) {
        if (t == tid && again && chunks == 1) {
          f(c * PL_THREADS, mine);
          continue;
        }
        const Tile x = tile_of(t);
        if (t == tid) mine = x;
        f(c * PL_THREADS, x);
      }
    }
  };
  auto steps_of = [&](int len) { return max((len + a.key_tile - 1) / a.key_tile, 1); };
  unsigned long long keys = 0;
  int longest = 0;
  each(false, [&](int, const Tile& x) {
    keys += a.columns ? steps_of(x.len) : x.len;
    longest = max(longest, x.len);
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    keys += __shfl_xor(keys, o);
    longest = max(longest, __shfl_xor(longest, o));
  }
  if (lane == 0 && keys) {
    atomicAdd(&s.keys, keys);
    atomicMax(&s.longest, longest);
  }
  __syncthreads();
  if (a.columns) {
    const unsigned long long all = s.keys;
    const unsigned long long S = max((all + a.columns - 1) / a.columns, 1ULL);
    const bool small = all >> 31 == 0;
    auto column_of = [&](unsigned long long step) { return small ? (int)((unsigned)step / (unsigned)S) : (int)(step / S); };
    unsigned long long done = 0;   // steps and units of the chunks before
    int units = 0;
    // sum of v over the threads before this one, and over all
    auto before = [&](auto v, auto* sums, auto& total) {
      auto sum = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const auto w = __shfl_up(sum, o);
        if (lane >= o) sum += w;
      }
      __syncthreads();   // (the last use of sums is over)
      if (lane == 63) sums[wave] = sum;
      __syncthreads();
      total = 0;
      sum -= v;
      for (int w = 0; w < PL_THREADS / 64; ++w) {
        if (w < wave) sum += sums[w];
        total += sums[w];
      }
      return sum;
    };
    for (int c = 0; c < chunks; ++c) {
      if (chunks > 1) tiles = load(c * PL_THREADS);
      const Tile x = tid < tiles ? (chunks == 1 ? mine : tile_of(tid)) : Tile{0, 0, 0, 0};
      const unsigned long long n = tid < tiles ? steps_of(x.len) : 0;
      unsigned long long steps;
      int pieces;
      const unsigned long long from = done + before(n, s.wave_steps, steps);
      const int p = n ? column_of(from + n - 1) - column_of(from) + 1 : 0;
      const int u0 = before(p, s.wave_sum, pieces);
      if (n) {
        int slot = -1;
        if (p > 1) {
          slot = atomicAdd(&s.slots, p);
          a.splits[atomicAdd(&s.n_splits, 1)] =
              ChunkSplit{c * PL_THREADS + x.r, x.tile, slot, p, s.row0[x.r], s.n[x.r], s.L[x.r], 0};
        }
        s.k0[tid] = x.k0;
        s.len[tid] = x.len;
        s.step[tid] = from;
        s.slot[tid] = slot;
      }
      s.unit[tid] = u0;
      __syncthreads();
      for (int i = tid; i < pieces; i += PL_THREADS) {
        int t = 0;   // the last tile with unit[t] <= i
#pragma unroll
        for (int st = PL_THREADS / 2; st > 0; st >>= 1)
          if (t + st < tiles && s.unit[t + st] <= i) t += st;
        const unsigned long long tile_from = s.step[t];
        const int w = column_of(tile_from) + i - s.unit[t];
        const unsigned long long col = w * S;
        // keys of the tile before the column, and up to its end
        const long long at0 = col > tile_from ? (long long)(col - tile_from) * a.key_tile : 0;
        const long long at1 = min((long long)s.len[t], (long long)(col + S - tile_from) * a.key_tile);
        const int r = request_of(t), slot = s.slot[t];
        a.units[units + i] = ChunkUnit{c * PL_THREADS + r, t - s.first[r], s.k0[t] + (int)at0, s.k0[t] + (int)at1,
                                       slot < 0 ? -1 : slot + i - s.unit[t], s.row0[r], s.n[r], s.L[r]};
        if (col >= tile_from) a.first[w] = units + i;   // (a column begins in one unit)
      }
      done += steps;
      units += pieces;
      __syncthreads();
    }
    for (int w = column_of(done + S - 1) + tid; w <= a.columns; w += PL_THREADS) a.first[w] = units;
    if (tid == 0) {
      a.status[0] = s.bits;
      a.status[1] = units;
      a.status[2] = s.n_splits;
      a.status[3] = 0;
    }
    return;
  }
  const int S = chunk_unit_keys(a, s.keys, all_tiles);
  const int shift = max(26 - __builtin_clz(min(S, s.longest) | 1), 0);   // lengths >> shift are below 64
  auto bucket = [&](int len) -> int { return PL_BUCKETS - 1 - min(len >> shift, PL_BUCKETS - 1); };
  each(true, [&](int, const Tile& x) {
    int q;
    const int p = chunk_pieces(x.len, S, a.key_tile, q);
    if (p > 1) atomicAdd(&s.hist[bucket(q)], p - 1);
    atomicAdd(&s.hist[bucket(x.len - (p - 1) * q)], 1);
  });
  __syncthreads();
  if (wave == 0) {   // exclusive prefix of the 64 buckets
    const int n = s.hist[lane];
    int v = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(v, o);
      if (lane >= o) v += w;
    }
    s.hist[lane] = v - n;
    if (lane == 63) a.status[1] = v;
  }
  __syncthreads();
  each(true, [&](int b0, const Tile& x) {
    int q;
    const int p = chunk_pieces(x.len, S, a.key_tile, q), b = b0 + x.r;
    const int row0 = s.row0[x.r], n = s.n[x.r], L = s.L[x.r];
    int slot = -1;
    if (p > 1) {
      slot = atomicAdd(&s.slots, p);
      a.splits[atomicAdd(&s.n_splits, 1)] = ChunkSplit{b, x.tile, slot, p, row0, n, L, 0};
    }
    for (int i = 0; i < p; ++i) {
      const int at0 = i * q, at1 = i == p - 1 ? x.len : at0 + q;
      const int at = atomicAdd(&s.hist[bucket(at1 - at0)], 1);
      a.units[at] = ChunkUnit{b, x.tile, x.k0 + at0, x.k0 + at1, slot < 0 ? -1 : slot + i, row0, n, L};
    }
  });
  __syncthreads();
  if (tid == 0) {
    a.status[0] = s.bits;
    a.status[2] = s.n_splits;
    a.status[3] = 0;
  }
}

}  // namespace
}  // namespace hspec
