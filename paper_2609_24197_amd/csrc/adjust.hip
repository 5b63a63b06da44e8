// Logits of a ragged batch of verification rows on their way to the choice: bias, penalties for what was said, a
// grammar's mask.  Row j of a request comes after its first j drafts, which count as said.
//
//   x = l + bias;  x = x > 0 ? x / rho : x rho where v was said or stands in the prompt;
//   x = x - (phi n + pi) where v was said n > 0 times;  x = -inf where the row's mask has no bit
//
// Bound by memory: the logits are read once and written once.  A workgroup takes a slice of the vocabulary and the rows
// of one request in turn: it counts the request's history into LDS for its slice alone (whole-number additions, so any
// order serves), keeps what a token's row-independent part comes to in registers, and each row is then one load, a few
// operations and one store per token, with the next row's loads under way.
#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

constexpr int AJ_THREADS = 256;
constexpr int AJ_VEC = 8;                     // tokens a thread takes side by side: a byte of the mask
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

// Slice blockIdx.x of the vocabulary, request blockIdx.y, part blockIdx.z of its rows.
template <class Tin, class Tout, int G>
__global__ void __launch_bounds__(AJ_THREADS) adjust_kernel(AdjustArgs a, int part) {
  constexpr int S = AJ_THREADS * AJ_VEC * G, GS = AJ_THREADS * AJ_VEC;
  __shared__ unsigned s_cnt[S];
  __shared__ int s_bias[S];   // entry of the bias list, from 1 on
  const int tid = threadIdx.x, b = blockIdx.y;
  if (blockIdx.x == gridDim.x - 1) {
    if (b == 0 && blockIdx.z == 0) check_call(a);
    return;
  }
  const int v0 = blockIdx.x * S;
  const ChunkRows rows = request_rows(a, b);
  const int j0 = blockIdx.z * part, j1 = min(j0 + part, rows.n);
  if (j0 >= j1) return;
  const Tin* src = static_cast<const Tin*>(a.logits) + (size_t)(rows.row0 + j0) * a.V;
  Tout* dst = static_cast<Tout*>(a.out) + (size_t)(rows.row0 + j0) * a.V;
  const int words = (a.V + 31) / 32;
  int v[G], left[G];   // first token of a group, and how many of the row are left there
#pragma unroll
  for (int g = 0; g < G; ++g) {
    v[g] = v0 + g * GS + tid * AJ_VEC;
    left[g] = a.V - v[g];
  }
  float n[G][AJ_VEC];        // the next row's logits and mask, on their way
  unsigned nbits[G];
  auto fetch = [&](int j) {
    const int r = rows.row0 + j;
    int m = -1;
    if (a.mask) m = a.mask_rows ? a.mask_rows[r] : r;
    const bool masked = m >= 0 && m < a.masks;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      nbits[g] = 0xff;
      if (left[g] <= 0) continue;
      load8(src + (size_t)(j - j0) * a.V + v[g], left[g], n[g]);
      if (masked) nbits[g] = reinterpret_cast<const uint8_t*>(a.mask + (size_t)m * words)[v[g] / 8];
    }
  };
  fetch(j0);

  for (int i = tid; i < S; i += AJ_THREADS) {
    s_cnt[i] = 0;
    s_bias[i] = 0;
  }
  const History h = history(a, b);
  const Penalties pen = penalties(a, b);
  __syncthreads();
  const int32_t* said = a.history + (size_t)b * a.max_hist;
  constexpr int U = 8;
  for (int i0 = 0; i0 < h.n; i0 += U * AJ_THREADS) {
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * AJ_THREADS + tid;
      id[u] = i < h.n ? said[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * AJ_THREADS + tid;
      const unsigned at = (unsigned)id[u] - (unsigned)v0;
      if (id[u] >= 0 && at < S) {
        if (i < h.old) atomicOr(&s_cnt[at], AJ_PROMPT);
        else atomicAdd(&s_cnt[at], 1u);
      }
    }
  }
  for (int j = tid; j < j0; j += AJ_THREADS) {   // (k = 0: j0 = 0)
    if (!a.draft_tokens) break;
    const int t = draft_id(a, b, j);
    const unsigned at = (unsigned)t - (unsigned)v0;
    if (t >= 0 && at < S) atomicAdd(&s_cnt[at], 1u);
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
  float bias[G][AJ_VEC], less[G][AJ_VEC];
  unsigned seen[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    seen[g] = 0;
#pragma unroll
    for (int e = 0; e < AJ_VEC; ++e) {
      const int at = g * GS + tid * AJ_VEC + e;
      const unsigned c = s_cnt[at];
      const int i = s_bias[at];
      seen[g] |= (c ? 1u : 0u) << e;
      less[g][e] = cost(c);
      bias[g][e] = i ? a.bias[(size_t)b * a.n_bias + i - 1] : 0.f;
    }
  }
  for (int j = j0; j < j1; ++j) {
    float x[G][AJ_VEC];
    unsigned bits[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      bits[g] = nbits[g];
#pragma unroll
      for (int e = 0; e < AJ_VEC; ++e) x[g][e] = n[g][e];
    }
    if (j + 1 < j1) fetch(j + 1);
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
      for (int e = 0; e < AJ_VEC; ++e) {
        float y = x[g][e] + bias[g][e];
        y *= seen[g] >> e & 1 ? (y > 0.f ? pen.inv_rho : pen.rho) : 1.f;
        y -= less[g][e];
        x[g][e] = bits[g] >> e & 1 ? y : -INFINITY;
      }
      if (left[g] > 0) store8(dst + (size_t)(j - j0) * a.V + v[g], left[g], x[g]);
    }
    if (a.draft_tokens && j + 1 < j1) {
      const int t = draft_id(a, b, j);
      const unsigned at = (unsigned)t - (unsigned)v0;
      if (t >= 0 && at < S && (int)(at % GS / AJ_VEC) == tid) {   // (this thread alone reads the token's count from here on)
        const float c = cost(s_cnt[at] += 1);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int e = 0; e < AJ_VEC; ++e)
            if (at == (unsigned)(g * GS + tid * AJ_VEC + e)) {
              less[g][e] = c;
              seen[g] |= 1u << e;
            }
      }
    }
  }
}

template <class Tin, class Tout, int G>
hipError_t launch_g(const AdjustArgs& a, hipStream_t s) {
  const int slices = (a.V + AJ_THREADS * AJ_VEC * G - 1) / (AJ_THREADS * AJ_VEC * G);
  // workgroups enough for the chip: the rows of a request are split where slices and requests make too few
  const long long wgs = (long long)slices * a.B;
  const int parts = (int)std::max(1LL, std::min<long long>(a.k + 1, 1024 / wgs));
  const int part = (a.k + parts) / parts;
  const dim3 grid(slices + 1, a.B, (a.k + part) / part);
  hipLaunchKernelGGL((adjust_kernel<Tin, Tout, G>), grid, dim3(AJ_THREADS), 0, s, a, part);
  return hipGetLastError();
}
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
