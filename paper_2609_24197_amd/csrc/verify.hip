// Which drafted tokens stand against the target's probabilities, and the token that follows them.
//
// Row j of a request holds the target's logits after j drafts.  With p_j = softmax(l_j / T) and q_j the
// distribution draft t_j came from (softmax(d_j / Td) over the drafter's vocabulary, or all on t_j):
//   n = the first j with not (u_j q_j(t_j) < p_j(t_j)), or the number of drafts;
//   next = argmax_v log max(p_n(v) - q_n(v), 0) + G(v),  q = 0 after the last draft
// (Gumbel-max over the residual distribution; over p_n where no residual is positive).  Greedy: t_j stands
// while it is the argmax of l_j, and next = argmax l_n.
//
// Bound by reading the logits.  Launch 1 takes pieces of rows to (maximum, sum of exponentials, argmax); launch 2
// joins them, decides n in every workgroup of a request, and reads row n once more for the choice.
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int VF_THREADS = 256;
constexpr int ST_BAD_TOKEN = 4;
constexpr int ST_NONFINITE = 8;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A logit over its temperature.  NaN counts as -inf and +inf (or what overflows) as the largest float; both flag.
__device__ __forceinline__ float scaled(float l, float inv_t, bool& bad) {
  const float x = l * inv_t;
  if (x <= FLT_MAX) return x + 0.f;   // (-0 becomes 0: they tie)
  bad = true;
  return x == x ? FLT_MAX : -INFINITY;
}

// (maximum, sum of 2^((x - maximum) log2 e)) of what a lane has seen.
struct Lse {
  float m = -INFINITY, s = 0.f;
  __device__ __forceinline__ void join(float m2, float s2) {
    const float mn = fmaxf(m, m2);
    const float ref = mn == -INFINITY ? 0.f : mn;
    s = s * __builtin_amdgcn_exp2f((m - ref) * LOG2E) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * LOG2E);
    m = mn;
  }
};

// Part of a row for one thread: f(first element, values, count) on 16-byte pieces, single elements at ragged ends.
// Rows begin at any element, so pieces start at the first aligned one.
template <class T, class F>
__device__ __forceinline__ void each_piece(const T* row, int e0, int e1, F f) {
  constexpr int N = 16 / sizeof(T);
  const int mis = (int)((reinterpret_cast<uintptr_t>(row + e0) / sizeof(T)) % N);
  const int a0 = min(e1, e0 + (mis ? N - mis : 0)), a1 = a0 + (e1 - a0) / N * N;
  float v[N];
  for (int e = a0 + (int)threadIdx.x * N; e < a1; e += VF_THREADS * N) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(row + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = x[i];
    } else {
      const bf16x8 x = ld8(row + e);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = bf2f(x[i]);
    }
    f(e, v, Int<N>{});
  }
  const int ends = (a0 - e0) + (e1 - a1);   // fewer than 2 N
  if ((int)threadIdx.x < ends) {
    const int e = (int)threadIdx.x < a0 - e0 ? e0 + threadIdx.x : a1 + (threadIdx.x - (a0 - e0));
    v[0] = to_f32(row[e]);
    f(e, v, Int<1>{});
  }
}

// Statistics of elements [e0, e1) of a row over the workgroup; thread 0 has the result.
template <class T, bool GREEDY>
__device__ __forceinline__ float4 row_stats(const T* row, int e0, int e1, float inv_t) {
  __shared__ float4 s_w[VF_THREADS / 64];
  Lse a;
  unsigned long long best = 0;
  bool bad = false;
  each_piece(row, e0, e1, [&](int e, float* v, auto n) {
    constexpr int N = decltype(n)::value;
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = scaled(v[i], inv_t, bad);
      mx = fmaxf(mx, v[i]);
    }
    if constexpr (GREEDY) {
      if (mx > a.m || best == 0) {   // (a thread's elements come in rising order: the first maximum stays)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const unsigned long long key = ((unsigned long long)score_ord(v[i]) << 32) | ~(unsigned)(e + i);
          best = key > best ? key : best;
        }
      }
      a.m = fmaxf(a.m, mx);
    } else {
      float s = 0.f;
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((v[i] - ref) * LOG2E);
      a.join(mx, s);
    }
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    if constexpr (GREEDY) {
      const unsigned long long k = ((unsigned long long)__shfl_xor((unsigned)(best >> 32), o) << 32) |
                                   __shfl_xor((unsigned)best, o);
      best = k > best ? k : best;
    } else {
      const float m2 = __shfl_xor(a.m, o), s2 = __shfl_xor(a.s, o);
      a.join(m2, s2);
    }
  }
  bad = __any(bad);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0)
    s_w[wave] = GREEDY ? float4{__uint_as_float((unsigned)(best >> 32)), __uint_as_float((unsigned)best), 0.f, bad ? 1.f : 0.f}
                       : float4{a.m, a.s, 0.f, bad ? 1.f : 0.f};
  __syncthreads();
  float4 r = s_w[0];
  if (threadIdx.x == 0) {
    Lse t;
    unsigned long long top = 0;
    float flag = 0.f;
    for (int w = 0; w < VF_THREADS / 64; ++w) {
      const float4 x = s_w[w];
      flag = fmaxf(flag, x.w);
      if constexpr (GREEDY) {
        const unsigned long long k = ((unsigned long long)__float_as_uint(x.x) << 32) | __float_as_uint(x.y);
        top = k > top ? k : top;
      } else {
        t.join(x.x, x.y);
      }
    }
    r = GREEDY ? float4{__uint_as_float((unsigned)(top >> 32)), __uint_as_float((unsigned)top), 0.f, flag}
               : float4{t.m, t.s, 0.f, flag};
  }
  return r;
}

__device__ __forceinline__ int2 piece_range(int n, int pieces, int p) {
  const int len = ((n + pieces - 1) / pieces + 255) / 256 * 256;
  return int2{min(n, p * len), min(n, (p + 1) * len)};
}

template <class T, bool GREEDY>
__global__ void __launch_bounds__(VF_THREADS) verify_stats(VerifyArgs a) {
  const int w = blockIdx.x;
  if (threadIdx.x == 0) {
    if (w == 0) a.status[0] = 0;
    for (int b = w; b < a.B; b += gridDim.x) {
      a.count[b] = 0;
      for (int i = 0; i < kVerifyKeys; ++i) a.keys[b * kVerifyKeys + i] = 0;
    }
  }
  const int nt = a.rows * a.pieces_t;
  if (w < nt) {
    const int r = w / a.pieces_t, p = w % a.pieces_t;
    if (a.cu && r >= a.cu[a.B]) return;
    const int2 e = piece_range(a.V, a.pieces_t, p);
    const float4 s = row_stats<T, GREEDY>(static_cast<const T*>(a.target) + (size_t)r * a.V, e.x, e.y, GREEDY ? 1.f : a.inv_t);
    if (threadIdx.x == 0) a.stat_t[w] = s;
  } else if constexpr (!GREEDY) {
    const int x = w - nt, r = x / a.pieces_d, p = x % a.pieces_d;
    const int b = r / a.k, j = r % a.k;
    if (a.cu && j >= chunk_rows(a.cu, b, a.rows, a.k + 1).n - 1) return;
    const int2 e = piece_range(a.Vd, a.pieces_d, p);
    const float4 s = row_stats<float, false>(a.draft + (size_t)r * a.Vd, e.x, e.y, a.inv_td);
    if (threadIdx.x == 0) a.stat_d[x] = s;
  }
}

// log(sum) of a row's pieces; flag: a value was not finite, or no value is above -inf.
__device__ __forceinline__ float join_pieces(const float4* s, int n, bool& flag) {
  Lse t;
  for (int i = 0; i < n; ++i) {
    const float4 x = s[i];
    t.join(x.x, x.y);
    flag |= x.w != 0.f;
  }
  flag |= t.m == -INFINITY;
  return t.m == -INFINITY ? -INFINITY : t.m + __builtin_amdgcn_logf(t.s) * LN2;
}
// x - lse, for rows of nothing but -inf too
__device__ __forceinline__ float log_prob(float x, float lse) { return x == -INFINITY ? -INFINITY : x - lse; }
__device__ __forceinline__ float exp_nat(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// One workgroup per (request, piece of the vocabulary); greedy takes one piece and needs no row.
template <class T, bool GREEDY>
__global__ void __launch_bounds__(VF_THREADS) verify_pick(VerifyArgs a) {
  __shared__ int s_n, s_flags, s_last;
  __shared__ float s_lse_p, s_lse_q;
  __shared__ unsigned long long s_key[VF_THREADS / 64][kVerifyKeys];
  const int b = blockIdx.x / a.pieces_r, piece = blockIdx.x % a.pieces_r;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  ChunkRows cr;
  if (a.cu) {
    cr = chunk_rows(a.cu, b, a.rows, a.k + 1);
  } else {
    cr.row0 = b * (a.k + 1);
    cr.n = a.k + 1;
    cr.ok = true;
  }
  if (!cr.ok && tid == 0) set_status(a.status, ST_BAD_ROWS);
  int32_t* out = a.tokens + (size_t)b * (a.k + 1);
  if (cr.n == 0) {   // a request without rows
    if (piece == 0) {
      for (int i = tid; i <= a.k; i += VF_THREADS) out[i] = -1;
      if (tid == 0) a.accepted[b] = 0;
    }
    return;
  }
  const int drafts = cr.n - 1;
  if (tid == 0) {
    s_n = drafts;
    s_flags = 0;
  }
  __syncthreads();
  // the first draft that does not stand
  for (int j0 = 0; j0 < drafts; j0 += VF_THREADS) {
    const int j = j0 + tid;
    bool stands = true;
    if (j < drafts) {
      const int d = a.draft_tokens[(size_t)b * a.k + j];
      const int t = d < 0 || d >= a.Vd ? -1 : a.d2t ? a.d2t[d] : d;
      stands = false;
      if (t >= 0 && t < a.V) {
        const float4* st = a.stat_t + (size_t)(cr.row0 + j) * a.pieces_t;
        if constexpr (GREEDY) {
          unsigned long long top = 0;
          for (int i = 0; i < a.pieces_t; ++i) {
            const unsigned long long k = ((unsigned long long)__float_as_uint(st[i].x) << 32) | __float_as_uint(st[i].y);
            top = k > top ? k : top;
          }
          stands = key_token(top) == t;
        } else {
          bool flag = false, ignore = false;
          const float lse = join_pieces(st, a.pieces_t, flag);
          const float x = scaled(to_f32(static_cast<const T*>(a.target)[(size_t)(cr.row0 + j) * a.V + t]), a.inv_t, ignore);
          const float p = exp_nat(log_prob(x, lse));
          float q = 1.f;
          if (a.draft) {
            const size_t r = (size_t)b * a.k + j;
            const float lq = join_pieces(a.stat_d + r * a.pieces_d, a.pieces_d, flag);
            q = exp_nat(log_prob(scaled(a.draft[r * a.Vd + d], a.inv_td, ignore), lq));
          }
          stands = a.u[(size_t)b * a.k + j] * q < p;
        }
      }
    }
    if (!stands) atomicMin(&s_n, j);
    __syncthreads();
    if (s_n < drafts) break;
  }
  __syncthreads();
  const int n = s_n;
  // flags of the rows that decided: their values, and the drafts' tokens
  for (int j = tid; j <= n; j += VF_THREADS) {
    int f = 0;
    const float4* st = a.stat_t + (size_t)(cr.row0 + j) * a.pieces_t;
    bool flag = false;
    if constexpr (GREEDY) {
      unsigned top = 0;
      for (int i = 0; i < a.pieces_t; ++i) {
        flag |= st[i].w != 0.f;
        top = max(top, __float_as_uint(st[i].x));
      }
      flag |= top == score_ord(-INFINITY);
    } else {
      const float lse = join_pieces(st, a.pieces_t, flag);
      if (j == n) s_lse_p = lse;
      if (a.draft && j < drafts) {
        const float lq = join_pieces(a.stat_d + ((size_t)b * a.k + j) * a.pieces_d, a.pieces_d, flag);
        if (j == n) s_lse_q = lq;
      }
    }
    if (flag) f |= ST_NONFINITE;
    if (j < drafts) {
      const int d = a.draft_tokens[(size_t)b * a.k + j];
      const int t = d < 0 || d >= a.Vd ? -1 : a.d2t ? a.d2t[d] : d;
      if (t < 0 || t >= a.V) f |= ST_BAD_TOKEN;
    }
    if (f && piece == 0) atomicOr(&s_flags, f);
  }
  __syncthreads();
  int next = -1;
  if constexpr (GREEDY) {
    unsigned long long top = 0;
    const float4* st = a.stat_t + (size_t)(cr.row0 + n) * a.pieces_t;
    for (int i = 0; i < a.pieces_t; ++i) {
      const unsigned long long k = ((unsigned long long)__float_as_uint(st[i].x) << 32) | __float_as_uint(st[i].y);
      top = k > top ? k : top;
    }
    next = key_token(top);
    if (tid == 0 && s_flags) set_status(a.status, s_flags);
  } else {
    const T* row = static_cast<const T*>(a.target) + (size_t)(cr.row0 + n) * a.V;
    const float* noise = a.gumbel + (size_t)b * a.V;
    const bool rejected = n < drafts;
    const float* drow = rejected && a.draft ? a.draft + ((size_t)b * a.k + n) * a.Vd : nullptr;
    int hot = -1;   // the draft that all of q is on
    if (rejected && !a.draft) {
      const int d = a.draft_tokens[(size_t)b * a.k + n];
      hot = d < 0 || d >= a.Vd ? -1 : a.d2t ? a.d2t[d] : d;
    }
    const float lse_p = s_lse_p, lse_q = drow ? s_lse_q : 0.f;
    unsigned long long best[kVerifyKeys] = {0, 0};
    bool bad_noise = false, bad_map = false, ignore = false;
    const int2 e = piece_range(a.V, a.pieces_r, piece);
    each_piece(row, e.x, e.y, [&](int v0, const float* x, auto cnt) {
      constexpr int N = decltype(cnt)::value;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int v = v0 + i;
        const float lp = log_prob(scaled(x[i], a.inv_t, ignore), lse_p);
        const float gn = noise[v];
        float own = lp + gn, rest = own;
        bool some = lp > -INFINITY && v != hot;
        if (drow) {
          int d = a.t2d ? a.t2d[v] : v < a.Vd ? v : -1;
          if (d < -1 || d >= a.Vd) {
            bad_map = true;
            d = -1;
          }
          if (d >= 0) {
            const float lq = log_prob(scaled(drow[d], a.inv_td, ignore), lse_q);
            if (lq > -INFINITY) {
              const float r = exp_nat(lp) - exp_nat(lq);
              some = r > 0.f;
              rest = __builtin_amdgcn_logf(r) * LN2 + gn;
            }
          }
        }
        if (!(own == own)) {
          bad_noise = bad_noise || !(gn == gn);
          own = -INFINITY;
        }
        if (!(rest == rest)) rest = -INFINITY;
        const unsigned long long k0 = some ? ((unsigned long long)score_ord(rest) << 32) | ~(unsigned)v : 0ull;
        const unsigned long long k1 = ((unsigned long long)score_ord(own) << 32) | ~(unsigned)v;
        best[0] = k0 > best[0] ? k0 : best[0];
        best[1] = k1 > best[1] ? k1 : best[1];
      }
    });
    const int f = (__any(bad_noise) ? ST_NONFINITE : 0) | (__any(bad_map) ? ST_BAD_TOKEN : 0);
    if (f && lane == 0) set_status(a.status, f);
#pragma unroll
    for (int i = 0; i < kVerifyKeys; ++i) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const unsigned long long k = ((unsigned long long)__shfl_xor((unsigned)(best[i] >> 32), o) << 32) |
                                     __shfl_xor((unsigned)best[i], o);
        best[i] = k > best[i] ? k : best[i];
      }
      if (lane == 0) s_key[wave][i] = best[i];
    }
    __syncthreads();
    if (tid < kVerifyKeys) {
      unsigned long long k = s_key[0][tid];
      for (int w = 1; w < VF_THREADS / 64; ++w) k = s_key[w][tid] > k ? s_key[w][tid] : k;
      if (k) atomicMax(a.keys + b * kVerifyKeys + tid, k);
      __threadfence();
    }
    __syncthreads();
    if (tid == 0) {
      if (s_flags) set_status(a.status, s_flags);
      s_last = atomicAdd(a.count + b, 1) == a.pieces_r - 1;
    }
    __syncthreads();
    if (!s_last) return;
    const unsigned long long k0 = __hip_atomic_load(a.keys + b * kVerifyKeys, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const unsigned long long k1 = __hip_atomic_load(a.keys + b * kVerifyKeys + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    next = key_token(k0 ? k0 : k1);
  }
  for (int i = tid; i <= a.k; i += VF_THREADS) {
    int t = i == n ? next : -1;
    if (i < n) {
      const int d = a.draft_tokens[(size_t)b * a.k + i];
      t = a.d2t ? a.d2t[d] : d;
    }
    out[i] = t;
  }
  if (tid == 0) a.accepted[b] = n;
}

template <class T>
hipError_t launch_typed(const VerifyArgs& a, hipStream_t s) {
  const bool greedy = a.u == nullptr;
  const long long wgs = (long long)a.rows * a.pieces_t + (!greedy && a.draft ? (long long)a.B * a.k * a.pieces_d : 0);
  auto stats = greedy ? verify_stats<T, true> : verify_stats<T, false>;
  hipLaunchKernelGGL(stats, dim3((unsigned)wgs), dim3(VF_THREADS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  auto pick = greedy ? verify_pick<T, true> : verify_pick<T, false>;
  hipLaunchKernelGGL(pick, dim3((unsigned)(a.B * (long long)a.pieces_r)), dim3(VF_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace

void verify_bounds(VerifyArgs& a) {
  // workgroups aimed for, and elements a piece has at least
  auto pieces = [](long long rows, int V) {
    const long long want = std::max(1LL, 4096 / std::max(rows, 1LL)), most = std::max(1, V / 4096);
    return (int)std::min(want, std::min(most, 64LL));
  };
  a.pieces_t = pieces(a.rows, a.V);
  a.pieces_d = pieces((long long)a.B * a.k, a.Vd);
  a.pieces_r = a.u ? pieces(a.B, a.V) : 1;
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  return a.f32 ? launch_typed<float>(a, s) : launch_typed<bf16>(a, s);
}

}  // namespace hspec
