// New tokens of a ragged batch on their way into the target's paged cache: per-head RMSNorm and RoPE of
// the q and k of a fused projection row [q heads | k heads | v heads], q out, K and V into their slots.
//
//   y = x rsqrt(mean(x^2) + eps) w;  (y_p, y_{p+D/2}) turned by pos theta^(-2p/D)
//
// Bound by memory: every element is read once and written once.  A lane holds E elements of both halves
// of a head, so a head's sum of squares is a shuffle over D / 2E lanes and a pair is turned in registers.
// The angle is taken in 64 bits: at position 10^6 an fp32 product is off by 2^-5 of a radian.
// 8000 rows of 80 heads, bf16, no norm: 63 us, 4.9 TB/s, what a copy of as many bytes takes; with the norm 65 (147 with
// the gains read and the heads divided anew each round); 1088 rows of 48 heads from fp32: 10.5 us.
#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int AP_THREADS = 256;
constexpr int AP_ROWS = 2;   // (with 1 and 4: 8000 bf16 rows of 48 heads 58 and 44 us, 45 here; 1088 fp32 rows 11.8 and 16, 11.7 on that card)

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

// AP_ROWS tokens per workgroup.  The last workgroup checks the call (no launch clears the status word).
template <class Tin, class T, bool NORM>
__global__ void __launch_bounds__(AP_THREADS) chunk_append_kernel(ChunkAppendArgs a, Turns turns) {
  constexpr int E = sizeof(Tin) == 2 && sizeof(T) == 2 ? 8 : 4;   // 16 bytes of the wider side per load or store
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a);
    return;
  }
  __shared__ float s_cs[AP_ROWS][64], s_sn[AP_ROWS][64];
  __shared__ long long s_slot[AP_ROWS];   // < 0: position not mapped (K and V skipped)
  __shared__ int s_pos[AP_ROWS];          // < 0: row of no request
  const int tid = threadIdx.x, wave = tid >> 6;
  const int r0 = blockIdx.x * AP_ROWS;
  const int D = a.D, half = D / 2;
  const int lph = half / E, heads = a.Hq + 2 * a.Hkv;   // lanes of a head (a power of two, at most 16)
  // A round of the workgroup is AP_THREADS / lph heads of consecutive rows; lanes past the end go through it with the
  // last row (shuffles stay whole).  Elements are on their way a round ahead, the first while positions, slots and
  // angles are found.
  const int i0 = tid % lph * E, ahead = AP_THREADS / lph, dt = ahead / heads, dh = ahead % heads;
  int nt = tid / lph / heads, nh = tid / lph % heads;   // row and head of the next round
  float x1[E], x2[E], n1[E], n2[E];
  auto fetch = [&]() {
    const Tin* src = static_cast<const Tin*>(a.qkv) + ((size_t)min(r0 + nt, a.T - 1) * heads + nh) * D + i0;
    load_e<Tin, E>(src, n1);
    load_e<Tin, E>(src + half, n2);
  };
  fetch();
  // a lane has the same columns of every head
  float gq[NORM ? 2 * E : 1], gk[NORM ? 2 * E : 1];
  if constexpr (NORM) {
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) {
      const int c = e < E ? i0 + e : half + i0 + e - E;
      gq[e] = a.qw[c];
      gk[e] = a.kw[c];
    }
  }
  for (int t = wave; t < AP_ROWS; t += AP_THREADS / 64) {   // a wave per token: its place, then its angles
    const int r = r0 + t, lane = tid & 63;
    const RowPlace at = row_place(a.cu, a.ctx_lens, a.B, a.T, a.max_new, r);
    int pos = -1;
    long long slot = -1;
    if (at.n > 0) {
      pos = chunk_pos(at.L, at.n, a.cap).L + at.i;
      const int pg = pos / a.ps;
      if (pg < a.max_pages) {
        const int id = a.page_table[(size_t)at.b * a.max_pages + pg];
        if (id >= 0 && id < a.num_pages) slot = (long long)id * a.ps + pos % a.ps;
      }
    }
    if (lane == 0) {
      s_pos[t] = pos;
      s_slot[t] = slot;
    }
    if (lane < half) {
      double rev = (double)pos * turns.per_pos[lane];
      rev -= rint(rev);
      float sn, cs;
      sincosf((float)(rev * 6.283185307179586476925286766559), &sn, &cs);
      s_cs[t][lane] = cs;
      s_sn[t][lane] = sn;
    }
  }
  __syncthreads();
  for (int w0 = 0; w0 < AP_ROWS * heads; w0 += ahead) {
    const int t = min(nt, AP_ROWS - 1), hd = nh;
    const bool live = nt < AP_ROWS;
    const int pos = s_pos[t];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x1[e] = n1[e];
      x2[e] = n2[e];
    }
    nt += dt;
    nh += dh;
    if (nh >= heads) {
      nh -= heads;
      ++nt;
    }
    if (w0 + ahead < AP_ROWS * heads) fetch();
    if (hd < a.Hq + a.Hkv) {
      if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += x1[e] * x1[e] + x2[e] * x2[e];
        for (int off = lph / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const float f = rsqrtf(ss / D + a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x1[e] = x1[e] * f * (hd < a.Hq ? gq[e] : gk[e]);
          x2[e] = x2[e] * f * (hd < a.Hq ? gq[E + e] : gk[E + e]);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float g1 = x1[e], g2 = x2[e], cs = s_cs[t][i0 + e], sn = s_sn[t][i0 + e];
        x1[e] = g1 * cs - g2 * sn;
        x2[e] = g2 * cs + g1 * sn;
      }
    }
    if (!live || pos < 0) continue;
    T* dst;
    if (hd < a.Hq) {
      dst = static_cast<T*>(a.q) + ((size_t)(r0 + t) * a.Hq + hd) * D + i0;
    } else {
      const long long slot = s_slot[t];
      if (slot < 0) continue;
      const int hk = hd - a.Hq;
      T* cache = static_cast<T*>(hk < a.Hkv ? a.k_cache : a.v_cache);
      dst = cache + ((size_t)slot * a.Hkv + (hk < a.Hkv ? hk : hk - a.Hkv)) * D + i0;
    }
    store_e<T, E>(dst, x1);
    store_e<T, E>(dst + half, x2);
  }
}

template <class Tin, class T>
hipError_t launch_typed(const ChunkAppendArgs& a, hipStream_t s) {
  Turns lt{};
  for (int p = 0; p < a.D / 2; ++p)   // (pair 0 turns by 1 whatever the base)
    lt.per_pos[p] = (p ? exp2(-2.0 * p / a.D * log2(a.rope_theta)) : 1.0) / 6.283185307179586476925286766559;
  const auto kern = a.qw ? chunk_append_kernel<Tin, T, true> : chunk_append_kernel<Tin, T, false>;
  hipLaunchKernelGGL(kern, dim3((a.T + AP_ROWS - 1) / AP_ROWS + 1), dim3(AP_THREADS), 0, s, a, lt);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_append(const ChunkAppendArgs& a, hipStream_t s) {
  if (a.D != 64 && a.D != 128) return hipErrorInvalidValue;
  if (a.in_f32) return a.out_f32 ? launch_typed<float, float>(a, s) : launch_typed<float, bf16>(a, s);
  return a.out_f32 ? launch_typed<bf16, float>(a, s) : launch_typed<bf16, bf16>(a, s);
}

}  // namespace hspec
