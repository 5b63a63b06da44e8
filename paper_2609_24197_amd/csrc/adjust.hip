// Logits of a ragged batch of verification rows on their way to the choice: bias, penalties for what was said, a
// grammar's mask.  Row j of a request comes after its first j drafts, which count as said.
//
//   x = l + bias;  x = x > 0 ? x / rho : x rho where v was said or stands in the prompt;
//   x = x - (phi n + pi) where v was said n > 0 times;  x = -inf where the row's mask has no bit
//
// Bound by memory: the logits are read once and written once.  A workgroup takes a slice of the vocabulary and the rows
// of one request in turn: it counts the request's history into LDS for its slice alone (whole-number additions, so any
// order serves), keeps what a token's row-independent part comes to in registers, and each row is then one load, a few
// operations and one store per token, with the next row's loads under way.  64 requests of 17 rows of 131072 bf16 logits:
// 120 us in the kernel, 4.8 TB/s (105 at its shortest); one row of 32000: 4.8.
#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int AJ_THREADS = 256;
constexpr int AJ_VEC = 8;                     // tokens a thread takes side by side: a byte of the mask
constexpr int AJ_PART = 64;                   // rows of a workgroup at most
constexpr unsigned AJ_PROMPT = 0x80000000u;   // in a token's count: it stands in the prompt
constexpr int ST_BAD_TOKEN = 4, ST_NONFINITE = 8;

// Penalties of a request; those outside their range count as none.
struct Penalties {
  float rho, inv_rho, phi, pi;
  bool ok;
};
__device__ __forceinline__ Penalties penalties(const AdjustArgs& a, int b) {
  const float far = 18446744073709551616.f;   // 2^64: sums and products with counts stay finite
  Penalties p{a.repetition ? a.repetition[b] : 1.f, 1.f, a.frequency ? a.frequency[b] : 0.f,
              a.presence ? a.presence[b] : 0.f, true};
  if (!(p.rho >= 1.f / far && p.rho <= far)) p.rho = 1.f, p.ok = false;
  if (!(fabsf(p.phi) <= far)) p.phi = 0.f, p.ok = false;
  if (!(fabsf(p.pi) <= far)) p.pi = 0.f, p.ok = false;
  p.inv_rho = 1.f / p.rho;
  return p;
}
// History of a request: `n` tokens, the first `old` of them its prompt.
struct History {
  int n, old;
  bool ok;
};
__device__ __forceinline__ History history(const AdjustArgs& a, int b) {
  History h{0, 0, true};
  if (!a.history) return h;
  const int n = a.hist_lens[b], old = a.prompt_lens ? a.prompt_lens[b] : 0;
  h.n = min(max(n, 0), a.max_hist);
  h.old = min(max(old, 0), h.n);
  h.ok = h.n == n && h.old == old;
  return h;
}
__device__ __forceinline__ ChunkRows request_rows(const AdjustArgs& a, int b) {
  if (a.cu) return chunk_rows(a.cu, b, a.rows, a.k + 1);
  return ChunkRows{b * (a.k + 1), a.k + 1, true};
}
// Target id of draft j of request b, -1 where it has none.
__device__ __forceinline__ int draft_id(const AdjustArgs& a, int b, int j) {
  int t = a.draft_tokens[(size_t)b * a.k + j];
  if ((unsigned)t >= (unsigned)a.Vd) return -1;
  if (a.d2t) t = a.d2t[t];
  return (unsigned)t < (unsigned)a.V ? t : -1;
}

// Checks of the whole call by one workgroup, which alone writes the status word.
__device__ void check_call(const AdjustArgs& a) {
  __shared__ int s_bits;
  if (threadIdx.x == 0) s_bits = 0;
  __syncthreads();
  int bits = 0;
  for (int b = threadIdx.x; b < a.B; b += AJ_THREADS) {
    if (!request_rows(a, b).ok) bits |= ST_BAD_ROWS;
    if (!history(a, b).ok) bits |= ST_BAD_CTX_LEN;
    if (!penalties(a, b).ok) bits |= ST_NONFINITE;
  }
  if (a.draft_tokens)
    for (int i = threadIdx.x; i < a.B * a.k; i += AJ_THREADS) {
      const int b = i / a.k, j = i % a.k;
      if (j + 1 < request_rows(a, b).n && draft_id(a, b, j) < 0) bits |= ST_BAD_TOKEN;
    }
  if (a.mask_rows) {
    const int top = a.cu ? min(max(a.cu[a.B], 0), a.rows) : a.rows;
    for (int r = threadIdx.x; r < top; r += AJ_THREADS)
      if (a.mask_rows[r] >= a.masks) bits |= ST_BAD_ROWS;
  }
  if (bits) atomicOr(&s_bits, bits);
  __syncthreads();
  if (threadIdx.x == 0) a.status[0] = s_bits;
}

// 8 logits from p on, of which those below `n` are in the row.  Rows begin at any element.
template <class T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[AJ_VEC]) {
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  constexpr int N = 16 / sizeof(T);
  if (n >= AJ_VEC) {
#pragma unroll
    for (int i = 0; i < AJ_VEC; i += N) {
      const Vec x = *reinterpret_cast<const Vec*>(p + i);
#pragma unroll
      for (int e = 0; e < N; ++e) v[i + e] = (float)x[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < AJ_VEC; ++e) v[e] = e < n ? (float)p[e] : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[AJ_VEC]) {
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  constexpr int N = 16 / sizeof(T);
  if (n >= AJ_VEC) {
#pragma unroll
    for (int i = 0; i < AJ_VEC; i += N) {
      Vec x;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (T)v[i + e];
      *reinterpret_cast<Vec*>(p + i) = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < AJ_VEC; ++e)
      if (e < n) p[e] = (T)v[e];
  }
}

// A thread's tokens of a row on their way: their logits and, per group of 8, their byte of the mask.
template <int G>
struct RowRegs {
  float x[G][AJ_VEC];
  unsigned bits[G];
};
// What stays the same over a request's rows, of the thread's tokens, but for the drafts that come to it.
template <int G>
struct TokenRegs {
  float bias[G][AJ_VEC], less[G][AJ_VEC];
  unsigned seen[G];
};

// Slice blockIdx.x of the vocabulary, request blockIdx.y, part blockIdx.z of its rows.
template <class Tin, class Tout, int G>
__global__ void __launch_bounds__(AJ_THREADS) adjust_kernel(AdjustArgs a, int part) {
  constexpr int S = AJ_THREADS * AJ_VEC * G, GS = AJ_THREADS * AJ_VEC;
  static_assert(AJ_THREADS == 256 && AJ_PART <= 64, "waves of s_before, bits of taken");
  __shared__ __align__(16) unsigned s_cnt[S];
  __shared__ __align__(16) int s_bias[S];   // entry of the bias list, from 1 on
  __shared__ int s_draft[AJ_PART], s_mask[AJ_PART];   // of each row: the draft that comes after it (-1: none), its line of the mask
  __shared__ int s_before[AJ_THREADS / 64];           // whether some of the rows are of a request before this one, too
  const int tid = threadIdx.x, b = blockIdx.y;
  if (blockIdx.x == gridDim.x - 1) {
    if (b == 0 && blockIdx.z == 0) check_call(a);
    return;
  }
  const int v0 = blockIdx.x * S;
  const ChunkRows rows = request_rows(a, b);
  const int j0 = blockIdx.z * part, j1 = min(j0 + part, rows.n);
  if (j0 >= j1) return;
  const Tin* src = static_cast<const Tin*>(a.logits) + (size_t)(rows.row0 + j0) * a.V + v0 + tid * AJ_VEC;
  Tout* dst = static_cast<Tout*>(a.out) + (size_t)(rows.row0 + j0) * a.V + v0 + tid * AJ_VEC;
  const int left = a.V - v0 - tid * AJ_VEC;   // tokens from this thread's first one on
  const bool whole = v0 + S <= a.V;           // (uniform)

  for (int i = tid; i < S / 4; i += AJ_THREADS) {
    reinterpret_cast<u32x4*>(s_cnt)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(s_bias)[i] = u32x4{0u, 0u, 0u, 0u};
  }
  for (int j = j0 + tid; j < j1; j += AJ_THREADS) {
    s_draft[j - j0] = a.draft_tokens && j + 1 < rows.n ? draft_id(a, b, j) : -1;
    int m = -1;
    if (a.mask) m = a.mask_rows ? a.mask_rows[rows.row0 + j] : rows.row0 + j;
    s_mask[j - j0] = m < a.masks ? m : -1;
  }
  // Where cu is bad, a row of several ranges is the first request's, so that one workgroup alone writes it (and, in place,
  // reads it).
  if (a.cu) {
    bool before = false;
#pragma unroll 4
    for (int i = tid; i < b; i += AJ_THREADS) {
      const RowsBefore r = rows_before(a.cu, i, b, a.rows, a.k + 1, rows.row0 + j0, j1 - j0);
      before |= r.from < r.to;
    }
    before = __any(before);
    if (tid % 64 == 0) s_before[tid / 64] = before;
  }
  const History h = history(a, b);
  const Penalties pen = penalties(a, b);
  __syncthreads();
  unsigned long long taken = 0;   // bit j - j0 of row j: another request's
  if (a.cu && (s_before[0] | s_before[1] | s_before[2] | s_before[3]))
    taken = rows_taken(a.cu, b, a.rows, a.k + 1, rows.row0 + j0, j1 - j0);
  const int32_t* said = a.history + (size_t)b * a.max_hist;
  auto count = [&](int id, int i) {
    const unsigned at = (unsigned)id - (unsigned)v0;
    if (id >= 0 && at < S) {
      if (i < h.old) atomicOr(&s_cnt[at], AJ_PROMPT);
      else atomicAdd(&s_cnt[at], 1u);
    }
  };
  typedef int Int4 __attribute__((ext_vector_type(4), aligned(4)));
  constexpr int U = 4;
  int at0 = 0;
  for (; at0 + 4 * U * AJ_THREADS <= h.n; at0 += 4 * U * AJ_THREADS) {
    Int4 id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = *reinterpret_cast<const Int4*>(said + at0 + (u * AJ_THREADS + tid) * 4);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) count(id[u][e], at0 + (u * AJ_THREADS + tid) * 4 + e);
  }
  for (; at0 < h.n; at0 += U * AJ_THREADS) {
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = said[min(at0 + u * AJ_THREADS + tid, h.n - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = at0 + u * AJ_THREADS + tid;
      if (i < h.n) count(id[u], i);
    }
  }
  if (a.draft_tokens) {   // the drafts of the parts before
    for (int j = tid; j < j0; j += AJ_THREADS) {
      const int t = draft_id(a, b, j);
      const unsigned at = (unsigned)t - (unsigned)v0;
      if (t >= 0 && at < S) atomicAdd(&s_cnt[at], 1u);
    }
  }
  for (int i = tid; i < a.n_bias; i += AJ_THREADS) {
    const int t = a.bias_ids[(size_t)b * a.n_bias + i];
    const unsigned at = (unsigned)t - (unsigned)v0;
    if (t >= 0 && at < S) atomicMax(&s_bias[at], i + 1);
  }
  __syncthreads();
  auto cost = [&](unsigned c) -> float {
    const unsigned said_n = c & ~AJ_PROMPT;
    return said_n ? fmaf(pen.phi, (float)said_n, pen.pi) : 0.f;
  };
  TokenRegs<G> k;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    k.seen[g] = 0;
#pragma unroll
    for (int e = 0; e < AJ_VEC; ++e) {
      const int at = g * GS + tid * AJ_VEC + e;
      const unsigned c = s_cnt[at];
      const int i = s_bias[at];
      k.seen[g] |= (c ? 1u : 0u) << e;
      k.less[g][e] = cost(c);
      k.bias[g][e] = i ? a.bias[(size_t)b * a.n_bias + i - 1] : 0.f;
    }
  }
  const int words = (a.V + 31) / 32;
  const uint8_t* mask = reinterpret_cast<const uint8_t*>(a.mask);
  // this thread's mask byte of row j, group g; where there is no mask, some byte that is there
  auto mask_at = [&](int m, int g) -> const uint8_t* {
    return m >= 0 ? mask + (size_t)m * words * 4 + (v0 + g * GS) / 8 + tid : reinterpret_cast<const uint8_t*>(a.logits);
  };
  auto adjusted = [&](RowRegs<G>& r) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < AJ_VEC; ++e) {
        float y = r.x[g][e] + k.bias[g][e];
        y *= k.seen[g] >> e & 1 ? (y > 0.f ? pen.inv_rho : pen.rho) : 1.f;
        y -= k.less[g][e];
        r.x[g][e] = r.bits[g] >> e & 1 ? y : -INFINITY;
      }
  };
  auto said_next = [&](int t) {   // the draft behind a row joins what was said
    const unsigned at = (unsigned)t - (unsigned)v0;
    if (t >= 0 && at < S && (int)(at % GS / AJ_VEC) == tid) {   // (this thread alone reads the token's count from here on)
      const float c = cost(s_cnt[at] += 1);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < AJ_VEC; ++e)
          if (at == (unsigned)(g * GS + tid * AJ_VEC + e)) {
            k.less[g][e] = c;
            k.seen[g] |= 1u << e;
          }
    }
  };
  if (whole && !taken) {
    // No branch around a load or store, so that a row's waits are for its own: with them 64 requests of 17 rows of 131072
    // take 195 us.
    auto fetch = [&](int j, RowRegs<G>& r) {
      const int i = min(j, j1 - 1) - j0, m = __builtin_amdgcn_readfirstlane(s_mask[i]);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        load8(src + (size_t)i * a.V + g * GS, AJ_VEC, r.x[g]);
        r.bits[g] = *mask_at(m, g) | (m >= 0 ? 0u : 0xffu);
      }
    };
    auto row = [&](int j, RowRegs<G>& r) {
      adjusted(r);
#pragma unroll
      for (int g = 0; g < G; ++g) store8(dst + (size_t)(j - j0) * a.V + g * GS, AJ_VEC, r.x[g]);
      said_next(__builtin_amdgcn_readfirstlane(s_draft[j - j0]));
    };
    RowRegs<G> r0, r1;
    fetch(j0, r0);
    for (int j = j0; j < j1; j += 2) {
      fetch(j + 1, r1);
      row(j, r0);
      if (j + 1 >= j1) break;
      fetch(j + 2, r0);
      row(j + 1, r1);
    }
    return;
  }
  // the last slice, or rows that are not all this request's
  for (int j = j0; j < j1; ++j) {
    if (taken >> (j - j0) & 1) {
      said_next(s_draft[j - j0]);
      continue;
    }
    RowRegs<G> r;
    const int m = __builtin_amdgcn_readfirstlane(s_mask[j - j0]);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      r.bits[g] = 0xff;
      if (left <= g * GS) continue;
      load8(src + (size_t)(j - j0) * a.V + g * GS, left - g * GS, r.x[g]);
      if (m >= 0) r.bits[g] = *mask_at(m, g);
    }
    adjusted(r);
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (left > g * GS) store8(dst + (size_t)(j - j0) * a.V + g * GS, left - g * GS, r.x[g]);
    said_next(s_draft[j - j0]);
  }
}

template <class Tin, class Tout, int G>
hipError_t launch_g(const AdjustArgs& a, hipStream_t s) {
  const int slices = (a.V + AJ_THREADS * AJ_VEC * G - 1) / (AJ_THREADS * AJ_VEC * G);
  // workgroups enough for the chip: the rows of a request are split where slices and requests make too few
  const long long wgs = (long long)slices * a.B;
  const int parts = (int)std::max<long long>((a.k + AJ_PART) / AJ_PART, std::min<long long>(a.k + 1, 1024 / wgs));
  const int part = (a.k + parts) / parts;
  const dim3 grid(slices + 1, a.B, (a.k + part) / part);
  hipLaunchKernelGGL((adjust_kernel<Tin, Tout, G>), grid, dim3(AJ_THREADS), 0, s, a, part);
  return hipGetLastError();
}
// One group of 8 tokens a thread where slices and requests are few: shorter workgroups, and more of them (one row of 32000:
// 3.6 us in a graph, 4.7 with two groups; 32 of them 5.0 and 6.1; 17 rows of each 17.6 and 18.3).  Two where they fill the
// chip anyway, which halves the counting of a history for each token (17 rows of 131072 of 16 requests: 26.7 us, 27.4 with
// one; of 32, 52.3 and 53.5; of 64, 113 either way; a row each of 16 requests, though, 7.4 and 6.2, of 64, 15.8 and 15.0).
template <class Tin, class Tout>
hipError_t launch_typed(const AdjustArgs& a, hipStream_t s) {
  return (long long)a.V * a.B <= (1 << 20) ? launch_g<Tin, Tout, 1>(a, s) : launch_g<Tin, Tout, 2>(a, s);
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, hipStream_t s) {
  if (a.in_f32) return a.out_f32 ? launch_typed<float, float>(a, s) : launch_typed<float, bf16>(a, s);
  return a.out_f32 ? launch_typed<bf16, float>(a, s) : launch_typed<bf16, bf16>(a, s);
}

}  // namespace hspec
