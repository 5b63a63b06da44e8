// What the kernels that put rows into a paged cache, or take them out, have in common: loads and stores of a lane's
// elements, RoPE's turns, the checks of a call.
#pragma once
#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int AP_THREADS = 256;

template <class T, int E>
__device__ __forceinline__ void load_e(const T* p, float (&v)[E]) {
  constexpr int N = 16 / sizeof(T);   // elements of a 16-byte load
#pragma unroll
  for (int i = 0; i < E; i += N) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    } else if constexpr (E >= 8) {
      const bf16x8 x = ld8(p + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i + e] = bf2f(x[e]);
    } else {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = bf2f(x[e]);
    }
  }
}
template <class T, int E>
__device__ __forceinline__ void store_e(T* p, const float (&v)[E]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
    typedef bf16 Vec __attribute__((ext_vector_type(E)));
    Vec x;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = f2bf(v[e]);
    *reinterpret_cast<Vec*>(p) = x;
  }
}

// Turns per position of each RoPE pair, theta^(-2p/D) / 2 pi: from the host, since 64-bit powers and divisions on the
// way to every token's angles sit on the critical path of a call of few tokens.
struct Turns {
  double per_pos[64];
};

inline Turns turns_of(int D, double theta) {
  Turns t{};
  for (int p = 0; p < D / 2; ++p)   // (pair 0 turns by 1 whatever the base)
    t.per_pos[p] = (p ? exp2(-2.0 * p / D * log2(theta)) : 1.0) / 6.283185307179586476925286766559;
  return t;
}

// Checks of the whole call by one workgroup, which alone writes the status word: the rows' division, the
// lengths, and the page of every position written.  A thread takes a request; requests of many pages are left to a
// wave each.
__device__ void check_call(const ChunkAppendArgs& a) {
  __shared__ int s_bits, s_big, s_list[AP_THREADS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_bits = 0;
  int bits = 0;
  auto page_ok = [&](int b, int pg) {
    const int id = a.page_table[(size_t)b * a.max_pages + pg];
    return id >= 0 && id < a.num_pages;
  };
  auto pages = [&](int b, int& first, int& last) {   // last < first: none
    const ChunkRows r = chunk_rows(a.cu, b, a.T, a.max_new);
    const ChunkPos p = chunk_pos(a.ctx_lens[b], r.n, a.cap);
    first = p.L / a.ps;
    last = r.n ? (min(p.L + r.n, a.cap) - 1) / a.ps : -1;
    return (r.ok ? 0 : ST_BAD_ROWS) | (p.ok ? 0 : ST_BAD_CTX_LEN);
  };
  constexpr int OWN = 4;
  for (int b0 = 0; b0 < a.B; b0 += AP_THREADS) {
    __syncthreads();
    if (tid == 0) s_big = 0;
    __syncthreads();
    if (b0 + tid < a.B) {
      int first, last;
      bits |= pages(b0 + tid, first, last);
      if (last - first >= OWN) {
        s_list[atomicAdd(&s_big, 1)] = b0 + tid;
      } else {
#pragma unroll
        for (int i = 0; i < OWN; ++i)
          if (first + i <= last && !page_ok(b0 + tid, first + i)) bits |= ST_BAD_PAGE;
      }
    }
    __syncthreads();
    for (int i = wave; i < s_big; i += AP_THREADS / 64) {
      int first, last;
      pages(s_list[i], first, last);
      for (int pg = first + lane; pg <= last; pg += 64)
        if (!page_ok(s_list[i], pg)) bits |= ST_BAD_PAGE;
    }
  }
  if (bits) atomicOr(&s_bits, bits);
  __syncthreads();
  if (tid == 0) a.status[0] = s_bits;
}

// Place of a row: its position (< 0: of no request) and its page's id (< 0: not mapped).  Every lane of a wave calls it.
struct RowSlot {
  int pos, page;
};
__device__ __forceinline__ RowSlot row_slot(const ChunkAppendArgs& a, int r) {
  const RowPlace at = row_place(a.cu, a.ctx_lens, a.B, a.T, a.max_new, r);
  RowSlot s{-1, -1};
  if (at.n > 0) {
    s.pos = chunk_pos(at.L, at.n, a.cap).L + at.i;
    const int pg = s.pos / a.ps;
    if (pg < a.max_pages) {
      const int id = a.page_table[(size_t)at.b * a.max_pages + pg];
      if (id >= 0 && id < a.num_pages) s.page = id;
    }
  }
  return s;
}

}  // namespace
}  // namespace hspec
