// New tokens of a ragged batch on their way into the target's paged cache: per-head RMSNorm and RoPE of
// the q and k of a fused projection row [q heads | k heads | v heads], q out, K and V into their slots.
//
//   y = x rsqrt(mean(x^2) + eps) w;  (y_p, y_{p+D/2}) turned by pos theta^(-2p/D)
//
// Bound by memory: every element is read once and written once.  A lane holds E elements of both halves
// of a head, so a head's sum of squares is a shuffle over D / 2E lanes and a pair is turned in registers.
// The angle is taken in 64 bits: at position 10^6 an fp32 product is off by 2^-5 of a radian.
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
    static_assert(E == 8, "one 16-byte store");
    bf16x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = f2bf(v[e]);
    *reinterpret_cast<bf16x8*>(p) = x;
  }
}

// Checks of the whole call by one workgroup, which alone writes the status word: the rows' division, the
// lengths, and the page of every position written.
__device__ void check_call(const ChunkAppendArgs& a) {
  __shared__ int s_bits;
  if (threadIdx.x == 0) s_bits = 0;
  __syncthreads();
  int bits = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = wave; b < a.B; b += AP_THREADS / 64) {
    const ChunkRows r = chunk_rows(a.cu, b, a.T, a.max_new);
    const ChunkPos p = chunk_pos(a.ctx_lens[b], r.n, a.cap);
    bits |= (r.ok ? 0 : ST_BAD_ROWS) | (p.ok ? 0 : ST_BAD_CTX_LEN);
    if (r.n == 0) continue;
    const int last = (min(p.L + r.n, a.cap) - 1) / a.ps;
    for (int pg = p.L / a.ps + lane; pg <= last; pg += 64) {
      const int id = a.page_table[(size_t)b * a.max_pages + pg];
      if (id < 0 || id >= a.num_pages) bits |= ST_BAD_PAGE;
    }
  }
  if (bits) atomicOr(&s_bits, bits);
  __syncthreads();
  if (threadIdx.x == 0) a.status[0] = s_bits;
}

// TB tokens per workgroup.  The last workgroup checks the call (no launch clears the status word).
template <class Tin, class T, int TB>
__global__ void __launch_bounds__(AP_THREADS) chunk_append_kernel(ChunkAppendArgs a, double log2_theta) {
  constexpr int E = sizeof(T) == 2 ? 8 : 4;
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a);
    return;
  }
  __shared__ float s_cs[TB][64], s_sn[TB][64];
  __shared__ long long s_slot[TB];   // < 0: position not mapped (K and V skipped)
  __shared__ int s_pos[TB];          // < 0: row of no request
  const int tid = threadIdx.x, wave = tid >> 6;
  const int r0 = blockIdx.x * TB;
  const int D = a.D, half = D / 2;
  for (int t = wave; t < TB; t += AP_THREADS / 64) {
    const int r = r0 + t;
    const int b = r < a.T ? row_request(a.cu, a.B, r) : -1;
    int pos = -1;
    long long slot = -1;
    if (b >= 0) {
      const ChunkRows cr = chunk_rows(a.cu, b, a.T, a.max_new);
      const int i = r - cr.row0;
      if (i >= 0 && i < cr.n) {
        pos = chunk_pos(a.ctx_lens[b], cr.n, a.cap).L + i;
        const int pg = pos / a.ps;
        if (pg < a.max_pages) {
          const int id = a.page_table[(size_t)b * a.max_pages + pg];
          if (id >= 0 && id < a.num_pages) slot = (long long)id * a.ps + pos % a.ps;
        }
      }
    }
    if ((tid & 63) == 0) {
      s_pos[t] = pos;
      s_slot[t] = slot;
    }
  }
  __syncthreads();
  for (int i = tid; i < TB * half; i += AP_THREADS) {
    const int t = i / half, p = i % half;
    const double inv = p ? exp2(-2.0 * (double)p / (double)D * log2_theta) : 1.0;   // (0 x log2(inf) is NaN)
    double phi = (double)s_pos[t] * inv;
    const double two_pi = 6.283185307179586476925286766559;
    phi -= two_pi * rint(phi / two_pi);
    float sn, cs;
    sincosf((float)phi, &sn, &cs);
    s_cs[t][p] = cs;
    s_sn[t][p] = sn;
  }
  __syncthreads();
  const int lph = half / E, heads = a.Hq + 2 * a.Hkv;   // lanes of a head (a power of two, at most 16)
  const int work = TB * heads * lph;
  for (int w0 = 0; w0 < work; w0 += AP_THREADS) {
    const int w = min(w0 + tid, work - 1);               // (lanes past the end repeat the last: shuffles stay whole)
    const int t = w / (heads * lph), hd = w / lph % heads, i0 = w % lph * E;
    const int pos = s_pos[t];
    const Tin* src = static_cast<const Tin*>(a.qkv) + ((size_t)min(r0 + t, a.T - 1) * heads + hd) * D + i0;
    float x1[E], x2[E];
    load_e<Tin, E>(src, x1);
    load_e<Tin, E>(src + half, x2);
    const float* gain = hd < a.Hq ? a.qw : a.kw;
    if (hd < a.Hq + a.Hkv) {
      float f = 1.f;
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += x1[e] * x1[e] + x2[e] * x2[e];
        for (int off = lph / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        f = rsqrtf(ss / D + a.eps);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float g1 = gain ? x1[e] * f * gain[i0 + e] : x1[e], g2 = gain ? x2[e] * f * gain[half + i0 + e] : x2[e];
        const float cs = s_cs[t][i0 + e], sn = s_sn[t][i0 + e];
        x1[e] = g1 * cs - g2 * sn;
        x2[e] = g2 * cs + g1 * sn;
      }
    }
    if (w0 + tid >= work || pos < 0) continue;
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
  const double lt = log2(a.rope_theta);
  if (a.T >= 2048)
    hipLaunchKernelGGL((chunk_append_kernel<Tin, T, 4>), dim3((a.T + 3) / 4 + 1), dim3(AP_THREADS), 0, s, a, lt);
  else
    hipLaunchKernelGGL((chunk_append_kernel<Tin, T, 1>), dim3(a.T + 1), dim3(AP_THREADS), 0, s, a, lt);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_append(const ChunkAppendArgs& a, hipStream_t s) {
  if (a.D != 64 && a.D != 128) return hipErrorInvalidValue;
  if (a.in_f32) return a.out_f32 ? launch_typed<float, float>(a, s) : launch_typed<float, bf16>(a, s);
  return a.out_f32 ? launch_typed<bf16, float>(a, s) : launch_typed<bf16, bf16>(a, s);
}

}  // namespace hspec
