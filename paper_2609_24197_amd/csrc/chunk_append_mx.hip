// New tokens of a ragged batch on their way into the 4-bit paged cache (mx.h), and cached positions on their way out.
//
//   append:  q = RoPE(RMSNorm_D(q) w_q), in fp32;  k the same in fp64, v as it is:
//            e = the smallest with max |y| < 7 2^e over 32 channels,  code = nearest of 0 .5 1 1.5 2 3 4 6 to |y| 2^-e
//   read:    code x 2^e
//
// Bound by memory: 8000 rows of 80 heads, bf16, no norm 63 to 65 us (5.0 TB/s, what a copy of as many bytes takes), 1088 rows
// of 48 heads from fp32 14; reading 66000 rows of 8 heads 77 us (4.3 TB/s).  A lane holds E channels of both halves of a head,
// so a block of 32 channels is 32 / E lanes of one half: its largest magnitude takes two or three shuffles, and a pair of RoPE
// is turned in registers.
//
// K is in 64 bits because a code is a step function: next to a border the last bits of a 32-bit norm and rotation choose
// between values 17 to 100 % apart, by how the sum of squares happens to be split over lanes.  In 64 bits the codes are
// those of the formula.  The rotation's sine and cosine in 64 bits are one lane's per pair and token, and the fp64 rate
// of the vector units is the fp32 one.
#include "append_rows.h"
#include "mx.h"

namespace hspec {
namespace {

// Rows a workgroup, two at every size: fewer suit few rows, more suit many.  With the norm, in a graph, for 1, 2 and 4 of
// them: 64 rows of 48 heads 6.2, 9.6 and 16.1 us; 1088 of them 13.7, 13.1 and 19.3; 2000 from bf16 25.8, 17.9 and 15.6; 8000
// of 80 heads 131, 98 and 89.
constexpr int AM_ROWS = 2;

// Codes of one lane's E channels of a block, and the block's scale byte; 32 / E neighbouring lanes share the block.
struct Quantised {
  unsigned codes, scale;
};
template <class R, int E>
__device__ __forceinline__ Quantised mx_quantise(const R (&y)[E]) {
  constexpr R top_of_32_bits = (R)3.4028235677973366e38;   // half a step past the largest fp32: what rounds to infinity
  R top = 0;
  bool wide = false;   // (a NaN too)
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const R v = y[e] < 0 ? -y[e] : y[e];
    wide |= !(v < top_of_32_bits);
    top = v > top ? v : top;
  }
  if (wide) top = (R)INFINITY;
#pragma unroll
  for (int off = 1; off < MX_BLOCK / E; off <<= 1) {
    const R o = __shfl_xor(top, off);
    top = o > top ? o : top;
  }
  Quantised r{0u, 255u};
  if (top < top_of_32_bits) {
    r.scale = mx_scale(top);
#pragma unroll
    for (int e = 0; e < E; ++e) r.codes |= mx_code(y[e], r.scale) << (4 * e);
  }
  return r;
}

template <class Tin, class T, bool NORM>
__global__ void __launch_bounds__(AP_THREADS) chunk_append_mx_kernel(ChunkAppendArgs a, Turns turns) {
  constexpr int E = sizeof(Tin) == 2 && sizeof(T) == 2 ? 8 : 4;   // 16 bytes of the wider side per load or store
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a);
    return;
  }
  __shared__ double s_cs[AM_ROWS][64], s_sn[AM_ROWS][64];
  __shared__ int s_page[AM_ROWS];   // < 0: position not mapped (K and V skipped)
  __shared__ int s_pos[AM_ROWS];    // < 0: row of no request
  const int tid = threadIdx.x, wave = tid >> 6;
  const int r0 = blockIdx.x * AM_ROWS;
  const int D = a.D, half = D / 2;
  const int lph = half / E, heads = a.Hq + 2 * a.Hkv;   // lanes of a head (a power of two, at most 16)
  // A round of the workgroup is AP_THREADS / lph heads of consecutive rows; lanes past the end go through it with the
  // last row (shuffles stay whole).  Elements are on their way a round ahead, the first while positions, pages and
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
  float gq[NORM ? 2 * E : 1], gk[NORM ? 2 * E : 1];   // a lane has the same columns of every head
  if constexpr (NORM) {
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) {
      const int c = e < E ? i0 + e : half + i0 + e - E;
      gq[e] = a.qw[c];
      gk[e] = a.kw[c];
    }
  }
  for (int t = wave; t < AM_ROWS; t += AP_THREADS / 64) {   // a wave per token: its place, then its angles
    const int lane = tid & 63;
    const RowSlot at = row_slot(a, r0 + t);
    if (lane == 0) {
      s_pos[t] = at.pos;
      s_page[t] = at.page;
    }
    if (lane < half) {
      double rev = (double)at.pos * turns.per_pos[lane], sn, cs;
      rev -= rint(rev);
      sincospi(2.0 * rev, &sn, &cs);
      s_cs[t][lane] = cs;
      s_sn[t][lane] = sn;
    }
  }
  __syncthreads();
  for (int w0 = 0; w0 < AM_ROWS * heads; w0 += ahead) {
    const int t = min(nt, AM_ROWS - 1), hd = nh;
    const bool live = nt < AM_ROWS;
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
    if (w0 + ahead < AM_ROWS * heads) fetch();
    if (hd < a.Hq) {
      if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += x1[e] * x1[e] + x2[e] * x2[e];
        for (int off = lph / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const float f = rsqrtf(ss / D + a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x1[e] = x1[e] * f * gq[e];
          x2[e] = x2[e] * f * gq[E + e];
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float g1 = x1[e], g2 = x2[e], cs = (float)s_cs[t][i0 + e], sn = (float)s_sn[t][i0 + e];
        x1[e] = g1 * cs - g2 * sn;
        x2[e] = g2 * cs + g1 * sn;
      }
      if (live && pos >= 0) {
        T* dst = static_cast<T*>(a.q) + ((size_t)(r0 + t) * a.Hq + hd) * D + i0;
        store_e<T, E>(dst, x1);
        store_e<T, E>(dst + half, x2);
      }
      continue;
    }
    const bool is_k = hd < a.Hq + a.Hkv;
    unsigned c1, c2, s1, s2;
    if (is_k) {
      double y1[E], y2[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y1[e] = x1[e];
        y2[e] = x2[e];
      }
      if constexpr (NORM) {
        double ss = 0.;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += y1[e] * y1[e] + y2[e] * y2[e];
        for (int off = lph / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const double f = 1. / sqrt(ss / D + (double)a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          y1[e] *= f * gk[e];
          y2[e] *= f * gk[E + e];
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double g1 = y1[e], g2 = y2[e], cs = s_cs[t][i0 + e], sn = s_sn[t][i0 + e];
        y1[e] = g1 * cs - g2 * sn;
        y2[e] = g2 * cs + g1 * sn;
      }
      const auto p = mx_quantise(y1), q = mx_quantise(y2);
      c1 = p.codes, s1 = p.scale, c2 = q.codes, s2 = q.scale;
    } else {
      const auto p = mx_quantise(x1), q = mx_quantise(x2);
      c1 = p.codes, s1 = p.scale, c2 = q.codes, s2 = q.scale;
    }
    const int page = s_page[t];
    if (!live || pos < 0 || page < 0) continue;
    const int hk = hd - a.Hq - (is_k ? 0 : a.Hkv), row = pos & (a.ps - 1);
    uint8_t* p = static_cast<uint8_t*>(is_k ? a.k_cache : a.v_cache) + ((size_t)page * a.Hkv + hk) * mx_head_bytes(a.ps, D);
    uint8_t* code = p + row * (D / 2) + i0 / 2;
    if constexpr (E == 8) {
      *reinterpret_cast<unsigned*>(code) = c1;
      *reinterpret_cast<unsigned*>(code + half / 2) = c2;
    } else {
      *reinterpret_cast<unsigned short*>(code) = (unsigned short)c1;
      *reinterpret_cast<unsigned short*>(code + half / 2) = (unsigned short)c2;
    }
    if (i0 % MX_BLOCK == 0) {
      uint8_t* scale = p + a.ps * (D / 2) + row * (D / MX_BLOCK) + i0 / MX_BLOCK;
      scale[0] = (uint8_t)s1;
      scale[half / MX_BLOCK] = (uint8_t)s2;
    }
  }
}

template <class Tin, class T>
hipError_t launch_typed(const ChunkAppendArgs& a, hipStream_t s) {
  const auto kern = a.qw ? chunk_append_mx_kernel<Tin, T, true> : chunk_append_mx_kernel<Tin, T, false>;
  hipLaunchKernelGGL(kern, dim3((a.T + AM_ROWS - 1) / AM_ROWS + 1), dim3(AP_THREADS), 0, s, a, turns_of(a.D, a.rope_theta));
  return hipGetLastError();
}

// -------------------------------------------------------------------------------- read

constexpr int RD_ROWS = 4;

// RD_ROWS rows per workgroup; a lane takes a word of 8 channels at a time, so that a wave's stores are whole lines.
template <class T, int D>
__global__ void __launch_bounds__(AP_THREADS) chunk_read_mx_kernel(ChunkAppendArgs a, T* k, T* v) {
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a);
    return;
  }
  __shared__ int s_page[RD_ROWS], s_pos[RD_ROWS];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int r0 = blockIdx.x * RD_ROWS;
  for (int t = wave; t < RD_ROWS; t += AP_THREADS / 64) {
    const RowSlot at = row_slot(a, r0 + t);
    if ((tid & 63) == 0) {
      s_pos[t] = at.pos;
      s_page[t] = at.page;
    }
  }
  __syncthreads();
  const int wpr = a.Hkv * D / 8;   // words of a row and tensor
  const size_t head_bytes = mx_head_bytes(a.ps, D);
  // a thread's next word, and which of the rows' k and v in turn it is of; counted on, not divided anew
  int q = tid / wpr, w = tid % wpr;
  const int dq = AP_THREADS / wpr, dw = AP_THREADS % wpr;
  constexpr int U = 4;   // words of a thread on their way together
  for (int i0 = tid; i0 < 2 * RD_ROWS * wpr; i0 += U * AP_THREADS) {
    unsigned code[U], scale[U];
    T* dst[U];
#pragma unroll
    for (int x = 0; x < U; ++x) {
      const int t = min(q >> 1, RD_ROWS - 1);
      const bool is_k = (q & 1) == 0;
      const int pos = s_pos[t], page = s_page[t];
      const int h = w / (D / 8), d = w % (D / 8) * 8, row = pos & (a.ps - 1);
      const uint8_t* p = static_cast<const uint8_t*>(is_k ? a.k_cache : a.v_cache) + ((size_t)max(page, 0) * a.Hkv + h) * head_bytes;
      code[x] = *reinterpret_cast<const unsigned*>(p + row * (D / 2) + d / 2);
      scale[x] = p[a.ps * (D / 2) + row * (D / MX_BLOCK) + d / MX_BLOCK];
      if (page < 0) code[x] = scale[x] = 0;   // (a position that is not mapped reads as zeros)
      dst[x] = q < 2 * RD_ROWS && pos >= 0 ? (is_k ? k : v) + ((size_t)(r0 + t) * a.Hkv + h) * D + d : nullptr;
      q += dq;
      w += dw;
      if (w >= wpr) {
        w -= wpr;
        ++q;
      }
    }
#pragma unroll
    for (int x = 0; x < U; ++x) {
      if (!dst[x]) continue;
      if constexpr (sizeof(T) == 4) {
        f32x4 lo, hi;
        mx_widen(code[x], scale[x], lo, hi);
        *reinterpret_cast<f32x4*>(dst[x]) = lo;
        *reinterpret_cast<f32x4*>(dst[x] + 4) = hi;
      } else {
        *reinterpret_cast<bf16x8*>(dst[x]) = mx_widen(code[x], scale[x]);
      }
    }
  }
}

}  // namespace

hipError_t launch_chunk_append_mx(const ChunkAppendArgs& a, hipStream_t s) {
  if (a.D != 64 && a.D != 128) return hipErrorInvalidValue;
  if (a.in_f32) return a.out_f32 ? launch_typed<float, float>(a, s) : launch_typed<float, bf16>(a, s);
  return a.out_f32 ? launch_typed<bf16, float>(a, s) : launch_typed<bf16, bf16>(a, s);
}

hipError_t launch_chunk_read_mx(const ChunkAppendArgs& a, void* k, void* v, hipStream_t s) {
  if (a.D != 64 && a.D != 128) return hipErrorInvalidValue;
  auto launch = [&](auto t, auto d) {
    typedef typename decltype(t)::type T;
    hipLaunchKernelGGL((chunk_read_mx_kernel<T, decltype(d)::value>), dim3((a.T + RD_ROWS - 1) / RD_ROWS + 1), dim3(AP_THREADS), 0, s,
                       a, static_cast<T*>(k), static_cast<T*>(v));
    return hipGetLastError();
  };
  if (a.out_f32) return a.D == 128 ? launch(std::common_type<float>{}, Int<128>{}) : launch(std::common_type<float>{}, Int<64>{});
  return a.D == 128 ? launch(std::common_type<bf16>{}, Int<128>{}) : launch(std::common_type<bf16>{}, Int<64>{});
}

}  // namespace hspec
