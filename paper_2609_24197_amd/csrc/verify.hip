// Which drafted tokens stand against the target's probabilities, and the token that follows them.
//
// Row j of a request holds the target's logits after j drafts.  With p_j = softmax(l_j / T) and q_j the
// distribution draft t_j came from (softmax(d_j / Td) over the drafter's vocabulary, or all on t_j):
//   n = the first j with not (u_j q_j(t_j) < p_j(t_j)), or the number of drafts;
//   next = argmax_v log max(p_n(v) - q_n(v), 0) + G(v),  q = 0 after the last draft
// (Gumbel-max over the residual distribution; over p_n where no residual is positive).  Greedy: t_j stands
// while it is the argmax of l_j, and next = argmax l_n.
//
// Bound by reading the logits.  Rows behind the first draft that does not stand are not needed, and which one that
// is comes out of the rows before it: the pieces of all rows are taken in the order of j by a grid that holds little
// more than one j of every request at a time; the workgroup that finishes a row decides its draft, and pieces of rows
// past a request's decision are left out.  Then row n is read once more for the choice.  64 requests x 16 drafts,
// 131072 bf16 logits: 162 us when every row was read first, now 67; where every draft stands 112 us (467 MB, 4.2 TB/s),
// greedy 71 (285 MB, 4.0 TB/s).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int VF_THREADS = 256;
constexpr int ST_BAD_TOKEN = 4;
constexpr int ST_NONFINITE = 8;
constexpr int VF_PIECE = kVerifyPiece;
constexpr int VF_GRID = 16384;    // (64 x 16 x 131072: 67 us, 77 with 4096, 74 with 8192)
constexpr float VF_LOWEST = -1074.f;   // log2 of the least probability that is not 0, as 64 bits have it
constexpr float VF_ERR = 1.25f * 0x1p-23f, VF_ERR0 = 20.f * 0x1p-23f;   // see verify_pick
constexpr float LN2 = 0.6931471805599453f;

// A logit as the definition wants it: NaN counts as -inf and +inf as the largest float; both flag.
__device__ __forceinline__ float clean(float l, bool& bad) {
  if (l <= FLT_MAX) return l;
  bad = true;
  return l == l ? FLT_MAX : -INFINITY;
}

// (maximum, sum of 2^((l - maximum) c)), c = log2(e) / T.  The difference is taken before the scale: of x = l c and a
// logarithm of their sum as large, it would carry the rounding of both (2^-24 of 40 / T).
struct Lse {
  float m = -INFINITY, s = 0.f;
  __device__ __forceinline__ void join(float m2, float s2, float c) {
    const float mn = fmaxf(m, m2);
    const float ref = mn == -INFINITY ? 0.f : mn;
    s = s * __builtin_amdgcn_exp2f((m - ref) * c) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * c);
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

__device__ __forceinline__ int2 piece_range(int n, int pieces, int p) {
  const int len = ((n + pieces - 1) / pieces + 255) / 256 * 256;
  return int2{min(n, p * len), min(n, (p + 1) * len)};
}

// A thread's part of a piece of at most VF_PIECE bytes on its way: 16-byte loads from the first aligned element on, and
// an element of the ragged ends.
constexpr int VF_VEC = VF_PIECE / (16 * VF_THREADS);
struct PieceRegs {
  u32x4 v[VF_VEC];
  float end;
  int a0, a1, e;   // aligned range, position of `end` (or -1)
};
template <class T>
__device__ __forceinline__ void load_piece(const T* row, int2 r, PieceRegs& x) {
  constexpr int N = 16 / sizeof(T);
  const int mis = (int)((reinterpret_cast<uintptr_t>(row + r.x) / sizeof(T)) % N);
  x.a0 = min(r.y, r.x + (mis ? N - mis : 0));
  x.a1 = x.a0 + (r.y - x.a0) / N * N;
#pragma unroll
  for (int i = 0; i < VF_VEC; ++i) {
    const int e = x.a0 + (i * VF_THREADS + (int)threadIdx.x) * N;
    if (e < x.a1) x.v[i] = *reinterpret_cast<const u32x4*>(row + e);
  }
  const int head = x.a0 - r.x, t = threadIdx.x;
  x.e = t < head ? r.x + t : t < head + (r.y - x.a1) ? x.a1 + t - head : -1;   // (fewer than 2 N of them)
  if (x.e >= 0) x.end = to_f32(row[x.e]);
}

// What a wave has of a piece: (maximum, sum) or the argmax key, and whether a value was not finite.
struct PieceStat {
  Lse l;
  unsigned long long key = 0;
  bool bad = false;
};
// f(value, place) for a thread's values, the ragged ends' last (place VF_END); BACK: from the last place to the first.
constexpr int VF_END = VF_VEC * 8;
template <class T, bool BACK, class F>
__device__ __forceinline__ void each_value(const PieceRegs& x, F f) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < VF_VEC; ++j) {
    const int i = BACK ? VF_VEC - 1 - j : j;
    if (x.a0 + (i * VF_THREADS + (int)threadIdx.x) * N < x.a1) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int q = BACK ? N - 1 - k : k;
        if constexpr (N == 4) f(__uint_as_float(x.v[i][q]), i * N + q);
        else f(__uint_as_float(q % 2 ? x.v[i][q / 2] & 0xffff0000u : x.v[i][q / 2] << 16), i * N + q);
      }
    }
  }
  if (x.e >= 0) f(x.end, VF_END);
}
// Two passes over the registers: the maximum (which a NaN comes through), then the sum against it or its first place.
// A wave with values that are not finite goes through its piece again by the rules of clean().
template <class T, bool GREEDY>
__device__ __forceinline__ PieceStat piece_stat(const PieceRegs& x, float c) {
  PieceStat s;
  float mx = -INFINITY;
  each_value<T, false>(x, [&](float v, int) { mx = __builtin_elementwise_maximum(mx, v); });
  const bool odd = __any(!(mx <= FLT_MAX));
  if (odd) {
    mx = -INFINITY;
    each_value<T, false>(x, [&](float v, int) { mx = fmaxf(mx, clean(v, s.bad)); });
  }
  const float ref = mx == -INFINITY ? 0.f : mx;
  s.l.m = mx;
  if constexpr (GREEDY) {
    // the first place of the maximum (-0 and 0 are equal); the ragged ends' element lies before or behind the others
    int at = INT_MAX;
    bool end = false;
    auto look = [&](float v, int place) {
      if (place == VF_END) end = v == mx;
      else at = v == mx ? place : at;
    };
    if (odd) each_value<T, true>(x, [&](float v, int place) { look(clean(v, s.bad), place); });
    else each_value<T, true>(x, look);
    constexpr int N = 16 / sizeof(T);
    if (at != INT_MAX) at = x.a0 + (at / N * VF_THREADS + (int)threadIdx.x) * N + at % N;
    if (end) at = min(at, x.e);
    if (at != INT_MAX) s.key = ((unsigned long long)score_ord(mx + 0.f) << 32) | ~(unsigned)at;
  } else if (odd) {
    each_value<T, false>(x, [&](float v, int) { s.l.s += __builtin_amdgcn_exp2f((clean(v, s.bad) - ref) * c); });
  } else {
    each_value<T, false>(x, [&](float v, int) { s.l.s += __builtin_amdgcn_exp2f((v - ref) * c); });
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    if constexpr (GREEDY) {
      const unsigned long long k = ((unsigned long long)__shfl_xor((unsigned)(s.key >> 32), o) << 32) | __shfl_xor((unsigned)s.key, o);
      s.key = k > s.key ? k : s.key;
    } else {
      const float m2 = __shfl_xor(s.l.m, o), s2 = __shfl_xor(s.l.s, o);
      s.l.join(m2, s2, c);
    }
  }
  s.bad = __any(s.bad);
  return s;
}

// ------------------------------------------------------------------------ rows, decisions

// Drafts of a request and its first row.
__device__ __forceinline__ ChunkRows request_rows(const VerifyArgs& a, int b) {
  if (a.cu) return chunk_rows(a.cu, b, a.rows, a.k + 1);
  return ChunkRows{b * (a.k + 1), a.k + 1, true};
}
// Target id of a drafted token, or -1.
__device__ __forceinline__ int target_id(const VerifyArgs& a, int d) {
  const int t = d < 0 || d >= a.Vd ? -1 : a.d2t ? a.d2t[d] : d;
  return t < a.V ? max(t, -1) : -1;
}
// log2 of a probability; of -inf, also in a row of nothing else, it is -inf.
__device__ __forceinline__ float log_prob(float l, const RowSum& r, float c) {
  return l == -INFINITY ? -INFINITY : __builtin_fmaf(l - r.m, c, -r.log_s);
}

__global__ void verify_init(VerifyArgs a) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i == 0) a.status[0] = 0;
  if (i < a.B * (a.k + 1)) a.count[(size_t)i * kVerifyLine] = 0;
  if (i < a.B) {
    const ChunkRows r = request_rows(a, i);
    a.n[i * kVerifyLine] = r.n - 1;   // (-1: no rows)
    a.req[i] = int2{r.row0, r.n - 1};
    a.done[i * kVerifyLine] = 0;
  }
}

// What a piece leaves is stored past the caches (agent scope) and waited for before its row's counter is raised, so
// that the last workgroup of a row, on any die, reads all of them.
__device__ __forceinline__ void publish(unsigned long long* p, unsigned long long v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  wait_vmcnt<0>();
}
__device__ __forceinline__ unsigned long long fetch(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// A piece as 64 bits: (maximum, sum) with the sum's sign as the flag of a value that was not finite, or the argmax key
// with the top bit of ~token (always 1: tokens are below 2^31) turned off by the flag.
constexpr unsigned long long KEY_BIT = 0x80000000ull;
__device__ __forceinline__ unsigned long long pack_lse(float m, float s, bool flag) {
  return ((unsigned long long)__float_as_uint(m) << 32) | __float_as_uint(flag ? -s : s);
}
__device__ __forceinline__ Lse unpack_lse(unsigned long long v, bool& flag) {
  const unsigned s = (unsigned)v;
  flag |= (s >> 31) != 0;
  return Lse{__uint_as_float((unsigned)(v >> 32)), __uint_as_float(s & 0x7fffffffu)};
}
__device__ __forceinline__ unsigned long long pack_key(unsigned long long key, bool flag) {
  if (!key) key = ((unsigned long long)score_ord(-INFINITY) << 32) | 0xffffffffu;   // (of no values)
  return flag ? key & ~KEY_BIT : key;
}
__device__ __forceinline__ unsigned long long unpack_key(unsigned long long v, bool& flag) {
  flag |= !(v & KEY_BIT);
  return v | KEY_BIT;
}

// Over the wave's lanes, of the pieces [0, n), n <= 64: a row's maximum and the log2 of its sum, and the flag.
__device__ __forceinline__ RowSum join_pieces(const unsigned long long* p, int n, float c, bool& flag) {
  const int lane = threadIdx.x & 63;
  Lse t;
  if (lane < n) t = unpack_lse(fetch(p + lane), flag);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(t.m, o), s2 = __shfl_xor(t.s, o);
    t.join(m2, s2, c);
  }
  flag = __any(flag) || t.m == -INFINITY;
  return RowSum{t.m, __builtin_amdgcn_logf(t.s)};
}

// Whether draft j of request b stands, and what the choice needs of its row (one wave).
template <class T, bool GREEDY>
__device__ __forceinline__ void decide(const VerifyArgs& a, int b, int j, const ChunkRows& cr) {
  const int lane = threadIdx.x & 63, drafts = cr.n - 1;
  const size_t row = (size_t)(cr.row0 + j);
  const int d = j < drafts ? a.draft_tokens[(size_t)b * a.k + j] : -1;
  const int t = target_id(a, d);
  bool flag = false, stands = false;
  VerifyRow r{};
  if constexpr (GREEDY) {
    unsigned long long top = 0;
    if (lane < a.pieces_t) top = unpack_key(fetch(a.stat_t + row * a.pieces_t + lane), flag);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long k = ((unsigned long long)__shfl_xor((unsigned)(top >> 32), o) << 32) | __shfl_xor((unsigned)top, o);
      top = k > top ? k : top;
    }
    flag = __any(flag) || (unsigned)(top >> 32) == score_ord(-INFINITY);
    r.top = key_token(top);
    stands = r.top == t;
  } else {
    bool ignore = false;
    // the drafted token's logits beside the pieces
    const float x = t >= 0 ? to_f32(static_cast<const T*>(a.target)[row * a.V + t]) : 0.f;
    const bool has_q = a.draft && j < drafts;
    const size_t dr = (size_t)b * a.k + j;
    const float y = has_q && t >= 0 ? a.draft[dr * a.Vd + d] : 0.f;
    const float u = j < drafts ? a.u[dr] : 0.f;
    r.p = join_pieces(a.stat_t + row * a.pieces_t, a.pieces_t, a.c_t, flag);
    float lq = 0.f;
    if (has_q) {
      r.q = join_pieces(a.stat_d + dr * a.pieces_d, a.pieces_d, a.c_d, flag);
      lq = log_prob(clean(y, ignore), r.q, a.c_d);
    }
    // u q < p by their logarithms, since 32 bits hold neither below 2^-126; below VF_LOWEST they count as 0
    const float lp = log_prob(clean(x, ignore), r.p, a.c_t);
    const float e = __builtin_amdgcn_exp2f((lq - lp) * 0.5f);   // (two factors, so that a small u meets no infinity first)
    stands = t >= 0 && lp >= VF_LOWEST && (u == 0.f || lq < VF_LOWEST || u * e * e < 1.f);
  }
  r.flags = (flag ? ST_NONFINITE : 0) | (j < drafts && t < 0 ? ST_BAD_TOKEN : 0);
  if (lane == 0) {
    a.row[(size_t)b * (a.k + 1) + j] = r;
    if (j < drafts && !stands) atomicMin(a.n + b * kVerifyLine, j);
  }
}

// Pieces of rows j of every request, for j in turn.
template <class T, bool GREEDY>
__global__ void __launch_bounds__(VF_THREADS) verify_rows(VerifyArgs a) {
  __shared__ unsigned long long s_stat[VF_THREADS / 64];   // as published
  __shared__ int s_need;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned pieces = a.pieces_t + (a.draft ? a.pieces_d : 0), per_j = a.B * pieces;
  const unsigned total = (a.k + 1) * per_j;   // (host: below 2^31)
  for (unsigned w = blockIdx.x; w < total; w += gridDim.x) {
    const int j = w / per_j, b = w % per_j / pieces, p = w % pieces;
    const int2 rq = a.req[b];
    // a request's decision so far (hearing of it later costs work, not the result): read once, so that all waves agree
    if (tid == 0) s_need = j <= __hip_atomic_load(a.n + b * kVerifyLine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const bool need = s_need && (p < a.pieces_t || j < rq.y);   // (the row after the last draft has no draft row)
    if (need) {
      PieceRegs x;
      PieceStat st;
      if (p < a.pieces_t) {
        load_piece(static_cast<const T*>(a.target) + (size_t)(rq.x + j) * a.V, piece_range(a.V, a.pieces_t, p), x);
        st = piece_stat<T, GREEDY>(x, a.c_t);
      } else if constexpr (!GREEDY) {
        load_piece(a.draft + ((size_t)b * a.k + j) * a.Vd, piece_range(a.Vd, a.pieces_d, p - a.pieces_t), x);
        st = piece_stat<float, false>(x, a.c_d);
      }
      if (lane == 0) s_stat[wave] = GREEDY ? pack_key(st.key, st.bad) : pack_lse(st.l.m, st.l.s, st.bad);
    }
    __syncthreads();
    if (need && wave == 0) {
      unsigned long long v = 0;
      bool bad = false;
      Lse t;
#pragma unroll
      for (int i = 0; i < VF_THREADS / 64; ++i) {
        if constexpr (GREEDY) {
          const unsigned long long k = unpack_key(s_stat[i], bad);
          v = k > v ? k : v;
        } else {
          const Lse l = unpack_lse(s_stat[i], bad);
          t.join(l.m, l.s, p < a.pieces_t ? a.c_t : a.c_d);
        }
      }
      v = GREEDY ? pack_key(v, bad) : pack_lse(t.m, t.s, bad);
      int last = 0;
      if (lane == 0) {
        publish(p < a.pieces_t ? a.stat_t + (size_t)(rq.x + j) * a.pieces_t + p
                               : a.stat_d + ((size_t)b * a.k + j) * a.pieces_d + (p - a.pieces_t), v);
        const int all = a.pieces_t + (a.draft && j < rq.y ? a.pieces_d : 0);
        last = atomicAdd(a.count + ((size_t)b * (a.k + 1) + j) * kVerifyLine, 1) == all - 1;
      }
      if (__builtin_amdgcn_readfirstlane(last)) decide<T, GREEDY>(a, b, j, ChunkRows{rq.x, rq.y + 1, true});
    }
  }
}

// ------------------------------------------------------------------------------ choice

// N values from any 4-byte boundary.
template <int N, class V>
__device__ __forceinline__ void load_n(const V* p, V (&v)[N]) {
  typedef V V4 __attribute__((ext_vector_type(4), aligned(4)));
  if constexpr (N == 1) {
    v[0] = p[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const V4 x = *reinterpret_cast<const V4*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = x[e];
    }
  }
}

// The best of some tokens: its score and token as a key (0: none), the most that its score can be without the
// roundings of 32 bits, and the most that any other's can be.
struct Pick {
  unsigned long long key;
  float hi, rival;
  __device__ __forceinline__ void join(unsigned long long k2, float h2, float r2) {
    rival = fmaxf(fmaxf(rival, r2), k2 > key ? hi : h2);
    hi = k2 > key ? h2 : hi;
    key = k2 > key ? k2 : key;
  }
  // Over the wave: neighbours, then pairs, quads, halves and rows of 16 lanes by moves between registers.
  template <int CTRL>
  __device__ __forceinline__ void join_dpp() {
    auto far = [](unsigned v) { return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true); };
    const unsigned long long k = ((unsigned long long)far((unsigned)(key >> 32)) << 32) | far((unsigned)key);
    const float h = __uint_as_float(far(__float_as_uint(hi))), r = __uint_as_float(far(__float_as_uint(rival)));
    join(k, h, r);
  }
  template <class SWAP>
  __device__ __forceinline__ void join_rows(SWAP swap) {
    const auto kh = swap((unsigned)(key >> 32)), kl = swap((unsigned)key), h = swap(__float_as_uint(hi)), r = swap(__float_as_uint(rival));
    *this = Pick{((unsigned long long)kh[0] << 32) | kl[0], __uint_as_float(h[0]), __uint_as_float(r[0])};
    join(((unsigned long long)kh[1] << 32) | kl[1], __uint_as_float(h[1]), __uint_as_float(r[1]));
  }
  __device__ __forceinline__ void join_wave() {
    join_dpp<0xb1>();    // lane ^ 1
    join_dpp<0x4e>();    // lane ^ 2
    join_dpp<0x141>();   // 7 - lane of 8
    join_dpp<0x140>();   // 15 - lane of 16
    join_rows([](unsigned v) { return __builtin_amdgcn_permlane16_swap(v, v, false, false); });
    join_rows([](unsigned v) { return __builtin_amdgcn_permlane32_swap(v, v, false, false); });
  }
  // Whether another token's score could reach this one's.  With ln(d + e) - ln d below 0.4, ln(d - e) lies above
  // ln d - 2 (ln(d + e) - ln d).
  __device__ __forceinline__ bool doubtful() const {
    if (!key) return true;
    const unsigned u = (unsigned)(key >> 32);
    const float best = __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u), up = hi - best;
    const float lo = best == INFINITY ? best : up < 0.4f ? best - 2.f * up : -INFINITY;
    return rival > -INFINITY && rival >= lo;
  }
};

// One workgroup per (request, piece of the vocabulary); greedy takes one piece and needs no row.
template <class T, bool GREEDY>
__global__ void __launch_bounds__(VF_THREADS) verify_pick(VerifyArgs a) {
  __shared__ int s_flags, s_last;
  __shared__ unsigned long long s_key[VF_THREADS / 64];
  __shared__ int s_who[VF_THREADS / 64];
  __shared__ Pick s_pick[VF_THREADS / 64];
  const int b = blockIdx.x / a.pieces_r, piece = blockIdx.x % a.pieces_r;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const ChunkRows cr = request_rows(a, b);
  const int n = max(a.n[b * kVerifyLine], 0);
  int32_t* out = a.tokens + (size_t)b * (a.k + 1);
  if (cr.n == 0) {   // a request without rows
    if (piece == 0) {
      for (int i = tid; i <= a.k; i += VF_THREADS) out[i] = -1;
      if (tid == 0) {
        a.accepted[b] = 0;
        if (!cr.ok) set_status(a.status, ST_BAD_ROWS);
      }
    }
    return;
  }
  const int drafts = cr.n - 1;
  const VerifyRow* rows = a.row + (size_t)b * (a.k + 1);
  const VerifyRow rn = rows[n];
  if (piece == 0) {   // flags of the rows that decided
    if (tid == 0) s_flags = cr.ok ? 0 : ST_BAD_ROWS;
    __syncthreads();
    int f = 0;
    for (int j = tid; j <= n; j += VF_THREADS) f |= rows[j].flags;
    if (f) atomicOr(&s_flags, f);
    __syncthreads();
    if (tid == 0 && s_flags) set_status(a.status, s_flags);
  }
  int next = -1;
  if constexpr (GREEDY) {
    next = rn.top;
  } else {
    const T* row = static_cast<const T*>(a.target) + (size_t)(cr.row0 + n) * a.V;
    const float* noise = a.gumbel + (size_t)b * a.V;
    const bool rejected = n < drafts;
    const float* drow = rejected && a.draft ? a.draft + ((size_t)b * a.k + n) * a.Vd : nullptr;
    // the draft that all of q is on
    const int hot = rejected && !a.draft ? target_id(a, a.draft_tokens[(size_t)b * a.k + n]) : -1;
    bool bad_noise = false, bad_map = false;
    const bool careful = (rn.flags & ST_NONFINITE) != 0;
    auto draft_of = [&](int v) {   // draft id of a target token, or -1
      const int d = a.t2d ? a.t2d[v] : v < a.Vd ? v : -1;
      return d < a.Vd ? max(d, -1) : -1;
    };
    // log2 of p is off by at most 2^-24 of (l - m) / T for the difference, for the scale and for the result, and what
    // the sum's logarithm is off by, so p by VF_ERR |log2 p| + VF_ERR0 of itself; the score is rounded once more.
    // log2(p - q) = log2 p + log2(1 - r), r = q / p, which holds where 32 bits hold neither p nor q.
    float best = -INFINITY;
    int at = -1;
    Pick pick{0, -INFINITY, -INFINITY};
    const int2 e = piece_range(a.V, a.pieces_r, piece);
    each_piece(row, e.x, e.y, [&](int v0, const float* x, auto cnt) {
      constexpr int N = decltype(cnt)::value;
      float gn[N], y[N];
      int d[N];
      load_n<N>(noise + v0, gn);
      if (drow) {
        if (a.t2d) load_n<N>(a.t2d + v0, d);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (!a.t2d) d[i] = v0 + i < a.Vd ? v0 + i : -1;
          if ((unsigned)(d[i] + 1) > (unsigned)a.Vd) {
            bad_map = true;
            d[i] = -1;
          }
          y[i] = d[i] >= 0 ? drow[d[i]] : -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        bool ignore = false;
        float lp = __builtin_fmaf(x[i] - rn.p.m, a.c_t, -rn.p.log_s);
        if (careful) lp = log_prob(clean(x[i], ignore), rn.p, a.c_t);
        const float err = __builtin_fmaf(fabsf(lp), VF_ERR, VF_ERR0);
        float lg = lp, up = lp;
        if (drow) {
          float lq = __builtin_fmaf(y[i] - rn.q.m, a.c_d, -rn.q.log_s);
          if (careful) lq = log_prob(clean(y[i], ignore), rn.q, a.c_d);
          // (of a difference below 0 the logarithm is NaN, which no comparison lets through)
          const float r = __builtin_amdgcn_exp2f(lq - lp), d1 = 1.f - r;
          lg += __builtin_amdgcn_logf(d1);
          up += __builtin_amdgcn_logf(__builtin_fmaf(1.f + r, err, d1));
        }
        const float sc = __builtin_fmaf(lg, LN2, gn[i]);
        const float top = __builtin_fmaf(up, LN2, gn[i]);
        const float hi = v0 + i == hot ? -INFINITY : __builtin_fmaf(fabsf(top), 0x1p-23f, top + err);
        bad_noise |= !(gn[i] == gn[i]);
        const bool better = sc > best && v0 + i != hot;
        pick.rival = fmaxf(pick.rival, better ? pick.hi : hi);
        pick.hi = better ? hi : pick.hi;
        best = better ? sc : best;
        at = better ? v0 + i : at;
      }
    });
    if (at >= 0) pick.key = ((unsigned long long)score_ord(best + 0.f) << 32) | ~(unsigned)at;
    pick.join_wave();
    const int f = (__any(bad_noise) ? ST_NONFINITE : 0) | (__any(bad_map) ? ST_BAD_TOKEN : 0);
    if (f && lane == 0) set_status(a.status, f);
    if (lane == 0) s_pick[wave] = pick;
    __syncthreads();
    unsigned long long* keys = a.keys + (size_t)b * verify_key_stride(a.pieces_r);
    if (tid == 0) {
#pragma unroll
      for (int w = 1; w < VF_THREADS / 64; ++w) pick.join(s_pick[w].key, s_pick[w].hi, s_pick[w].rival);
      publish(keys + 2 * piece, pick.key);
      publish(keys + 2 * piece + 1, ((unsigned long long)__float_as_uint(pick.hi) << 32) | __float_as_uint(pick.rival));
      s_last = atomicAdd(a.done + b * kVerifyLine, 1) == a.pieces_r - 1;
    }
    __syncthreads();
    if (!s_last) return;
    pick = Pick{0, -INFINITY, -INFINITY};
    if (lane < a.pieces_r) {   // (at most 64)
      const unsigned long long v = fetch(keys + 2 * lane + 1);
      pick = Pick{fetch(keys + 2 * lane), __uint_as_float((unsigned)(v >> 32)), __uint_as_float((unsigned)v)};
    }
    pick.join_wave();
    if (!pick.doubtful()) {
      next = key_token(pick.key);
    } else {
      // Rare: scores that lie closer together than 32 bits tell (about 10^-5 of the choices), or no positive difference.
      // The row once more in 64 (0.46 ms at 131072 tokens and 32000 of the drafter's).
      auto sum_of = [&](auto value, int count, double m, double c) {
        double t = 0.;
        for (int v = tid; v < count; v += VF_THREADS) t += exp2((value(v) - m) * c);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
        __syncthreads();
        if (lane == 0) s_key[wave] = (unsigned long long)__double_as_longlong(t);
        __syncthreads();
        t = 0.;
#pragma unroll
        for (int w = 0; w < VF_THREADS / 64; ++w) t += __longlong_as_double((long long)s_key[w]);
        return t;
      };
      bool ignore = false;
      auto target = [&](int v) { return (double)clean(to_f32(row[v]), ignore); };
      auto draft = [&](int d) { return (double)clean(drow[d], ignore); };
      // (p alone: the sum changes no order)
      const double sp = drow ? sum_of(target, a.V, rn.p.m, a.c64_t) : 1.;
      const double sq = drow ? sum_of(draft, a.Vd, rn.q.m, a.c64_d) : 1.;
      for (int own = 0; own < 2; ++own) {   // (own: no difference is positive)
        double hi = -INFINITY;
        int who = INT_MAX;
        for (int v = tid; v < a.V; v += VF_THREADS) {
          double p = exp2((target(v) - rn.p.m) * a.c64_t) / sp;
          const int d = !own && drow ? draft_of(v) : -1;
          if (d >= 0) p -= exp2((draft(d) - rn.q.m) * a.c64_d) / sq;
          const double sc = log(p) + noise[v];   // (NaN below 0)
          if (sc > hi && (own || v != hot)) {
            hi = sc;
            who = v;
          }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const double h2 = __shfl_xor(hi, o);
          const int w2 = __shfl_xor(who, o);
          if (h2 > hi || (h2 == hi && w2 < who)) {
            hi = h2;
            who = w2;
          }
        }
        __syncthreads();
        if (lane == 0) {
          s_key[wave] = (unsigned long long)__double_as_longlong(hi);
          s_who[wave] = who;
        }
        __syncthreads();
        for (int w = 0; w < VF_THREADS / 64; ++w) {
          const double h2 = __longlong_as_double((long long)s_key[w]);
          if (h2 > hi || (h2 == hi && s_who[w] < who)) {
            hi = h2;
            who = s_who[w];
          }
        }
        next = who == INT_MAX ? 0 : who;
        if (who != INT_MAX) break;
      }
    }
  }
  for (int i = tid; i <= a.k; i += VF_THREADS)
    out[i] = i < n ? target_id(a, a.draft_tokens[(size_t)b * a.k + i]) : i == n ? next : -1;
  if (tid == 0) a.accepted[b] = n;
}

template <class T>
hipError_t launch_typed(const VerifyArgs& a, hipStream_t s) {
  const bool greedy = a.u == nullptr;
  hipLaunchKernelGGL(verify_init, dim3((a.B * (a.k + 1) + 255) / 256), dim3(256), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  const long long items = (long long)(a.k + 1) * a.B * (a.pieces_t + (a.draft ? a.pieces_d : 0));
  auto rows = greedy ? verify_rows<T, true> : verify_rows<T, false>;
  hipLaunchKernelGGL(rows, dim3((unsigned)std::min(items, (long long)VF_GRID)), dim3(VF_THREADS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  auto pick = greedy ? verify_pick<T, true> : verify_pick<T, false>;
  hipLaunchKernelGGL(pick, dim3((unsigned)(a.B * (long long)a.pieces_r)), dim3(VF_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  VerifyArgs x = a;
  if (!a.u) x.pieces_r = 1;
  return a.f32 ? launch_typed<float>(x, s) : launch_typed<bf16>(x, s);
}

}  // namespace hspec
