// Causal attention of a ragged chunk of new tokens over the paged cache that already holds them.
//
//   o[r, h] = sum_s p_s V[s],  p = softmax over visible s of scale q[r, h] . K[s],
//   visible: max(0, pos - window + 1) <= s <= pos = ctx_len + (r - first row of the request)
//
// A workgroup takes one KV head and a tile of 32 NW (token, query head of the group) rows of one request, and
// walks a range of the request's keys.  A wave owns 32 of those rows as the columns of
//   S^T [keys x rows] = K Q^T   and   O^T [D x rows] += V^T P^T,
// 32 x 32 products: S^T leaves a lane with 16 keys of one row per 32-key block, so the running maximum needs one
// exchange between the wave's halves per tile, the running sum none until the end, and P^T is already in the
// layout of the second product's operand if V^T is read with its keys in the same order (they are summed over, so
// any order serves).  K and V tiles stream into LDS by direct DMA, the next tile while one is multiplied; in a page
// a wave's 16 rows are consecutive, so a tile costs a wave one page id.
//
// Three kernels: the plan (one workgroup: checks, list of units with the longest first, clears), the units, and
// the merge of rows whose keys were split.  Few rows and long caches are split over keys so that the chip is full;
// pieces are merged in key order, so results do not depend on timing.
//
// fp32 storage takes the fp32 matrix products (32 x 32 x 2), so nothing is rounded below 32 bits.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
#define LDS_AS __attribute__((address_space(3)))
#define GLB_AS __attribute__((address_space(1)))

// Source of K/V rows whose page id is outside the pool, and of tile rows no unit sees.
static __device__ __align__(16) const unsigned char zero_row[512] = {};

// Softmax reference maximum: raised, and O and the sum rescaled, only when a tile exceeds it by more than this
// many powers of two; probabilities then stay below 2^8.
constexpr float CHUNK_SLACK = 8.f;

template <class T, int D, int NW, int KT>
struct Chunk {
  static constexpr int NT = 64 * NW;
  static constexpr int ROWS = 32 * NW;
  static constexpr int EPC = 16 / sizeof(T);       // elements per 16-byte piece
  static constexpr int CPR = D / EPC;              // pieces per K/V row
  static constexpr int NB = KT / 32;               // 32-key blocks per tile
  static constexpr int NDB = D / 32;               // 32-wide d blocks of the output
  static constexpr int TILE = KT * D;
  static constexpr int WROWS = KT / NW;            // tile rows a wave fills
  static constexpr int GR = WROWS < 16 ? WROWS : 16;   // of them in one page for certain
  static constexpr int NG = WROWS / GR;
  static constexpr int NI = GR * CPR / 64;         // DMA instructions per group and tensor
  static_assert(KT % 32 == 0 && GR * CPR % 64 == 0 && WROWS % GR == 0, "tile shape");
};

// Element offset of (row, column d) in a K/V tile: 16-byte piece c of row r lives at piece c ^ f(r).  f makes the
// 16 rows a K fragment read touches at once, and the 4 rows x 64 bytes of a transposing V read, distinct bank groups.
template <class T, int CPR>
__device__ __forceinline__ int kv_off(int row, int d) {
  constexpr int EPC = 16 / sizeof(T);
  int f;
  if constexpr (CPR == 32) f = row & 15;
  else if constexpr (CPR == 16) f = ((row & 3) << 2) | ((row >> 2) & 3);
  else f = (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  return (row * CPR + ((d / EPC) ^ f)) * EPC + d % EPC;
}

// max over the two lanes l, l ^ 32
__device__ __forceinline__ float half_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// 8 keys x 32 d of V^T as the first operand: element j is key 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4.
template <int CPR>
__device__ __forceinline__ bf16x8 v_frag(const bf16* sV, int s, int db, int lane) {
  const int row = 16 * s + 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int d = db * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(sV + kv_off<bf16, CPR>(row, d)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(sV + kv_off<bf16, CPR>(row + 8, d)));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Whether any of n values in LDS is infinite or NaN (the whole wave gets the answer).
template <class T>
__device__ __forceinline__ bool tile_odd(const T* t, int n, int lane) {
  bool bad = false;
#pragma unroll 4
  for (int i = lane * (16 / (int)sizeof(T)); i < n; i += 64 * (16 / (int)sizeof(T))) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(t + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bad |= (x[e] & 0x7f800000u) == 0x7f800000u;
      if constexpr (sizeof(T) == 2) bad |= (x[e] & 0x7f80u) == 0x7f80u;
    }
  }
  return __any(bad);
}

// One unit's rows of one KV head.
template <class T, int D, int NW, int KT>
__device__ __forceinline__ void chunk_unit(const ChunkAttnArgs& a, const ChunkUnit& u, int h, T* st0, T* st1) {
  using C = Chunk<T, D, NW, KT>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NQ = F32 ? D / 8 : D / 16;        // 16-byte pieces of a row per lane
  typedef typename std::conditional<F32, f32x4, bf16x8>::type Frag;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, l32 = lane & 31;
  const int lps = 31 - __builtin_clz(a.ps);
  const int g = a.Hq / a.Hkv;
  const T* Kc = static_cast<const T*>(a.k_cache);
  const T* Vc = static_cast<const T*>(a.v_cache);
  const int row_elems = a.Hkv * D;
  const int R = u.n * g;                        // rows of the request
  const int c0 = u.tile * C::ROWS + wave * 32;  // first row of this wave
  const bool live = c0 < R;
  const int c = c0 + l32;
  const bool real = c < R;
  const int i_tok = real ? c / g : u.n - 1;
  const int hq = h * g + (real ? c - i_tok * g : 0);
  const size_t q_off = ((size_t)(u.row0 + i_tok) * a.Hq + hq) * D;
  // keys a column sees: [lo, hi); keys that any or all columns of the wave see
  const int t_first = live ? c0 / g : 0, t_last = live ? min(c0 + 31, R - 1) / g : 0;
  const int back = a.window > 0 ? a.window - 1 : INT_MAX;   // (positions are far below 2^31)
  auto sees_from = [&](int tok) { return max(u.L + tok - back, 0); };
  auto sees_to = [&](int tok) { return min(min(u.L + tok + 1, a.cap), u.k1); };
  const int lo = sees_from(i_tok), hi = real ? sees_to(i_tok) : INT_MIN;
  const int any_lo = sees_from(t_first), any_hi = sees_to(t_last);
  const int all_lo = sees_from(t_last), all_hi = sees_to(t_first);
  // first key any row of the unit sees: rows before it in the tile are not read
  const int k_min = max(u.k0, sees_from(u.tile * C::ROWS / g));

  Frag qf[NQ];
#pragma unroll
  for (int s = 0; s < NQ; ++s) {
    const int d = F32 ? 8 * s + 4 * hf : 16 * s + 8 * hf;
    if (real) {
      qf[s] = *reinterpret_cast<const Frag*>(static_cast<const T*>(a.q) + q_off + d);
    } else {
#pragma unroll
      for (int e = 0; e < C::EPC; ++e) qf[s][e] = (T)0.f;
    }
  }

  const int ntiles = u.k1 > u.k0 ? (u.k1 - u.k0 + KT - 1) / KT : 0;
  const int32_t* ptab = a.page_table + (size_t)u.b * a.max_pages;
  // page ids of this wave's row groups of tile ti (loaded a tile ahead of their use)
  auto load_pids = [&](int ti, int (&pid)[C::NG]) {
#pragma unroll
    for (int n = 0; n < C::NG; ++n) {
      const int key = u.k0 + ti * KT + wave * C::WROWS + n * C::GR;
      const bool any = key + C::GR > k_min && key < u.k1;
      pid[n] = any ? ptab[key >> lps] : -1;
    }
  };
  // DMA of tile ti into a stage: K rows, then V rows
  auto issue = [&](int ti, T* sb, const int (&pids)[C::NG]) {
#pragma unroll
    for (int n = 0; n < C::NG; ++n) {
      const int r0 = wave * C::WROWS + n * C::GR;
      const int key0 = u.k0 + ti * KT + r0;
      const int pid = __builtin_amdgcn_readfirstlane(pids[n]);
      const bool any = key0 + C::GR > k_min && key0 < u.k1;
      const bool good = any && pid >= 0 && pid < a.num_pages;
      if (any && !good && lane == 0) set_status(a.status, ST_BAD_PAGE);
      const size_t base = good ? (((size_t)pid << lps) + (key0 & (a.ps - 1))) * row_elems + h * D : 0;
      const T* kp = good ? Kc + base : reinterpret_cast<const T*>(zero_row);
      const T* vp = good ? Vc + base : reinterpret_cast<const T*>(zero_row);
      const int stride = good ? row_elems : 0;
      // rows outside the visible range repeat one inside it (they are masked, and a stale slot may hold NaN)
      const int first = max(k_min - key0, 0), last = max(min(u.k1 - key0, C::GR) - 1, 0);
#pragma unroll
      for (int i = 0; i < C::NI; ++i) {
        const int rr = (i * 64 + lane) / C::CPR, slot = (i * 64 + lane) % C::CPR;
        const int piece = kv_off<T, C::CPR>(r0 + rr, slot * C::EPC) / C::EPC - (r0 + rr) * C::CPR;   // stored here
        const int off = min(max(rr, first), last) * stride + piece * C::EPC;
        T* dst = sb + r0 * D + i * 64 * C::EPC;
        __builtin_amdgcn_global_load_lds((const GLB_AS void*)(kp + off), (LDS_AS void*)dst, 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const GLB_AS void*)(vp + off), (LDS_AS void*)(dst + C::TILE), 16, 0, 0);
      }
    }
  };

  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db) o[db] = zero16();
  float m_run = -INFINITY, l_run = 0.f;

  auto compute = [&](int ti, const T* sb) {
    const T* sK = sb;
    const T* sV = sb + C::TILE;
    const int base = u.k0 + ti * KT;
    if (!live || base >= any_hi || base + KT <= any_lo) return;   // (uniform) no key of the tile is visible here
    f32x16 st[C::NB];
#pragma unroll
    for (int kb = 0; kb < C::NB; ++kb) st[kb] = zero16();
#pragma unroll
    for (int s = 0; s < NQ; ++s)
#pragma unroll
      for (int kb = 0; kb < C::NB; ++kb) {
        const Frag kf = *reinterpret_cast<const Frag*>(
            sK + kv_off<T, C::CPR>(kb * 32 + l32, F32 ? 8 * s + 4 * hf : 16 * s + 8 * hf));
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            st[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[s][e], st[kb], 0, 0, 0);
        } else {
          st[kb] = mma32(kf, qf[s], st[kb]);
        }
      }

    const bool full = base + KT <= all_hi && base >= all_lo;
    bool odd = false;
    if (!full) {
#pragma unroll
      for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = base + kb * 32 + 8 * (i / 4) + 4 * hf + i % 4;
          if (key < lo || key >= hi) st[kb][i] = -INFINITY;
        }
      // Values of V that are not finite: a key that a row does not see has weight 0 in the product, and 0 x NaN
      // would reach the row all the same.  Here they are taken out of the product and added to the rows that see
      // them, as sums that overflow (a NaN as +inf and -inf).
      odd = tile_odd(sV, C::TILE, lane);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kb][i]);
    mx = half_max(mx) * a.scale_log2;
    if (__any(mx > m_run + CHUNK_SLACK)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < C::NDB; ++db) o[db] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][i], a.scale_log2, -m_use));
        st[kb][i] = e;
        l_run += e;
      }

    if constexpr (F32) {
#pragma unroll
      for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = kb * 32 + 8 * (i / 4) + 4 * hf + i % 4;
#pragma unroll
          for (int db = 0; db < C::NDB; ++db) {
            float v = sV[kv_off<T, C::CPR>(row, db * 32 + l32)];
            if (odd) {
              const float sees = base + row >= lo && base + row < hi ? FLT_MAX : 0.f;
              const bool fin = fabsf(v) < INFINITY;
              o[db] += __builtin_amdgcn_mfma_f32_32x32x2f32(fin || v < 0.f ? 0.f : FLT_MAX, sees, zero16(), 0, 0, 0);
              o[db] += __builtin_amdgcn_mfma_f32_32x32x2f32(fin || v > 0.f ? 0.f : -FLT_MAX, sees, zero16(), 0, 0, 0);
              if (!fin) v = 0.f;
            }
            o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, st[kb][i], o[db], 0, 0, 0);
          }
        }
    } else {
      // P enters the second product as bf16 (2^-9 relative to each weight, like the V it multiplies); the sum above
      // takes the unrounded weights
#pragma unroll
      for (int s = 0; s < 2 * C::NB; ++s) {
        bf16x8 pf;
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[j] = f2bf(st[s / 2][8 * (s & 1) + j]);
#pragma unroll
        for (int db = 0; db < C::NDB; ++db) {
          bf16x8 vf = v_frag<C::CPR>(sV, s, db, lane);
          if (odd) {
            s16x8 bits = __builtin_bit_cast(s16x8, vf), up, dn, sees;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const bool fin = (bits[j] & 0x7f80) != 0x7f80, nan = !fin && (bits[j] & 0x7f);
              const int key = base + 16 * s + 8 * (j / 4) + 4 * hf + j % 4;
              up[j] = (short)(!fin && (nan || bits[j] >= 0) ? 0x7f7f : 0);   // the largest bf16
              dn[j] = (short)(!fin && (nan || bits[j] < 0) ? 0xff7f : 0);
              sees[j] = (short)(key >= lo && key < hi ? 0x7f7f : 0);
              if (!fin) bits[j] = 0;
            }
            o[db] += mma32(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, sees), zero16());
            o[db] += mma32(__builtin_bit_cast(bf16x8, dn), __builtin_bit_cast(bf16x8, sees), zero16());
            vf = __builtin_bit_cast(bf16x8, bits);
          }
          o[db] = mma32(vf, pf, o[db]);
        }
      }
    }
  };

  int pids[C::NG];
  load_pids(0, pids);
  if (ntiles > 0) issue(0, st0, pids);
  if (ntiles > 1) load_pids(1, pids);
  auto step = [&](int ti, T* mine, T* other) {
    wait_vmcnt<0>();
    wg_barrier();   // every wave's part of tile ti has landed, and every wave has left the other stage
    if (ti + 1 < ntiles) issue(ti + 1, other, pids);
    if (ti + 2 < ntiles) load_pids(ti + 2, pids);
    compute(ti, mine);
  };
  for (int t0 = 0; t0 < ntiles; t0 += 2) {
    step(t0, st0, st1);
    if (t0 + 1 < ntiles) step(t0 + 1, st1, st0);
  }

  // lane holds O[row l32][d = 32 db + 8 (i / 4) + 4 hf + i % 4]
  const float l = half_sum(l_run);
  if (!real) return;
  if (u.slot < 0) {
    const float inv = hi > lo ? 1.f / l : 0.f;   // (a row that sees no key is zero)
    T* dst = static_cast<T*>(a.o) + q_off + 4 * hf;
#pragma unroll
    for (int db = 0; db < C::NDB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v = {o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
        v *= inv;
        if constexpr (F32) *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * q) = v;
        else *reinterpret_cast<bf16x4*>(dst + 32 * db + 8 * q) = bf16x4{f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
      }
  } else {
    const size_t pr = ((size_t)u.slot * a.Hkv + h) * C::ROWS + wave * 32 + l32;
    float* po = a.part_o + pr * D + 4 * hf;
#pragma unroll
    for (int db = 0; db < C::NDB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(po + 32 * db + 8 * q) =
            f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
    if (hf == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = float2{m_run, l};
  }
}

template <class T, int D, int NW, int KT>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
chunk_attn_kernel(ChunkAttnArgs a) {
  using C = Chunk<T, D, NW, KT>;
  __shared__ __align__(16) T st0[2 * C::TILE];   // two stages, so that the compiler can tell the one being read
  __shared__ __align__(16) T st1[2 * C::TILE];   // from the one whose DMA is in flight
  __shared__ int s_item[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_items = min(a.status[1], a.max_units) * a.Hkv;
  // Items go by class (item mod 8): a class's items share KV heads and its workgroups a die's L2.  A workgroup's
  // first item is its own index; the next come from its class's counter, then from the other classes'.
  // Each claim goes out at the start of an item and is looked at at its end.
  const int grid = gridDim.x;
  const int cls = blockIdx.x % kChunkClasses;
  auto item_of = [&](int c, int ticket) -> int {
    const long long it = ((long long)ticket + (grid - c + kChunkClasses - 1) / kChunkClasses) * kChunkClasses + c;
    return it < n_items ? (int)it : -1;
  };
  auto counter = [&](int c) { return a.queue + c * kChunkQueueStride; };
  // lanes of wave 0: an item of any class, or -1
  auto steal = [&]() -> int {
    for (;;) {
      int c = (cls + lane) % kChunkClasses, t = INT_MAX - grid;
      if (lane < kChunkClasses) t = __hip_atomic_load(counter(c), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const unsigned long long some = __ballot(lane < kChunkClasses && item_of(c, t) >= 0);
      if (!some) return -1;
      c = (cls + __builtin_ctzll(some)) % kChunkClasses;
      int got = 0;
      if (lane == 0) got = atomicAdd(counter(c), 1);
      const int it = item_of(c, __builtin_amdgcn_readfirstlane(got));
      if (it >= 0) return it;
    }
  };
  int item = blockIdx.x < n_items ? (int)blockIdx.x : -1;
  for (int turn = 0; item >= 0; turn ^= 1) {
    int ticket = 0;
    if (tid == 0 && n_items > grid) ticket = atomicAdd(counter(cls), 1);
    const ChunkUnit u = a.units[item / a.Hkv];
    const int h = item % a.Hkv;
    chunk_unit<T, D, NW, KT>(a, u, h, st0, st1);
    if (n_items <= grid) break;
    if (wave == 0) {
      int it = item_of(cls, __builtin_amdgcn_readfirstlane(ticket));
      if (it < 0) it = steal();
      if (lane == 0) s_item[turn] = it;
    }
    __syncthreads();   // the next item is known; every wave is done with this one
    item = __builtin_amdgcn_readfirstlane(s_item[turn]);
  }
}

// ------------------------------------------------------------------------------- plan

constexpr int PL_THREADS = 1024;
constexpr int PL_BUCKETS = 64;

struct PlanLds {
  int first[PL_THREADS + 1];          // tiles before each request of the chunk
  int row0[PL_THREADS], n[PL_THREADS], L[PL_THREADS];
  int wave_sum[PL_THREADS / 64];
  unsigned long long keys;            // keys of all tiles
  int longest, slots, n_splits, bits;
  int hist[PL_BUCKETS];
};

struct TileKeys {
  int k0, k1;   // key range, k0 a multiple of the key tile; k1 <= k0: no key
};
__device__ __forceinline__ TileKeys tile_keys(const ChunkAttnArgs& a, int g, int tile, int n, int L) {
  const int c0 = tile * a.tile_rows;
  const int t0 = c0 / g, t1 = (int)min((long long)c0 + a.tile_rows, (long long)n * g) - 1;
  TileKeys r;
  r.k1 = min(L + t1 / g + 1, a.cap);
  r.k0 = a.window > 0 ? max(L + t0 - a.window + 1, 0) / a.key_tile * a.key_tile : 0;
  return r;
}

// One workgroup lists the units.  Every tile of rows has len keys; tiles longer than S = max(min_split, all keys
// x Hkv / target) are cut into ceil(len / S) even pieces, so the pieces of all tiles number at most target / Hkv
// more than the tiles, and the split ones twice that (what the workspace holds).  Units are written longest first
// (64 classes of length), which keeps the queue's tail short.
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

  // Requests [c0, c0 + 1024): rows, lengths and tile counts into LDS.  Returns the chunk's tiles.
  auto load = [&](int c0) -> int {
    __syncthreads();
    const int b = c0 + tid;
    int nt = 0;
    if (b < a.B) {
      const ChunkRows r = chunk_rows(a.cu, b, a.T, a.max_new);
      const ChunkPos p = chunk_pos(a.ctx_lens[b], r.n, a.cap);
      if (!r.ok || !p.ok) atomicOr(&s.bits, (r.ok ? 0 : ST_BAD_ROWS) | (p.ok ? 0 : ST_BAD_CTX_LEN));
      s.row0[tid] = r.row0;
      s.n[tid] = r.n;
      s.L[tid] = p.L;
      nt = (int)(((long long)r.n * g + a.tile_rows - 1) / a.tile_rows);
    }
    int v = nt;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(v, o);
      if (lane >= o) v += w;
    }
    if (lane == 63) s.wave_sum[wave] = v;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += s.wave_sum[w];
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
  int tiles = 0;
  unsigned long long keys = 0;
  int longest = 0;
  for (int c = 0; c < chunks; ++c) {
    tiles = load(c * PL_THREADS);
    for (int t = tid; t < tiles; t += PL_THREADS) {
      const int r = request_of(t);
      const TileKeys k = tile_keys(a, g, t - s.first[r], s.n[r], s.L[r]);
      const int len = max(k.k1 - k.k0, 0);
      keys += len;
      longest = max(longest, len);
    }
  }
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
  // keys per unit, in whole key tiles
  const unsigned long long per = (s.keys * a.Hkv + a.target - 1) / a.target;
  const int S = (int)(((per < (unsigned long long)a.min_split ? (unsigned long long)a.min_split
                                                              : min(per, 1ull << 30)) + a.key_tile - 1) / a.key_tile * a.key_tile);
  const int top = min(S, s.longest) + 1;
  auto pieces_of = [&](int len, int& q) -> int {
    if (len <= S) {
      q = max(len, 1);
      return 1;
    }
    const int p = (int)(((long long)len + S - 1) / S);
    q = ((len + p - 1) / p + a.key_tile - 1) / a.key_tile * a.key_tile;
    return (len + q - 1) / q;
  };
  auto bucket = [&](int len) -> int { return PL_BUCKETS - 1 - (int)((long long)min(len, top - 1) * PL_BUCKETS / top); };
  auto each = [&](auto f) {
    for (int c = 0; c < chunks; ++c) {
      if (chunks > 1) tiles = load(c * PL_THREADS);
      for (int t = tid; t < tiles; t += PL_THREADS) {
        const int r = request_of(t), tile = t - s.first[r];
        const TileKeys k = tile_keys(a, g, tile, s.n[r], s.L[r]);
        int q;
        const int p = pieces_of(max(k.k1 - k.k0, 0), q);
        f(c * PL_THREADS + r, r, tile, k, q, p);
      }
    }
  };
  each([&](int, int, int, const TileKeys& k, int q, int p) {
    const int len = max(k.k1 - k.k0, 0);
    if (p > 1) atomicAdd(&s.hist[bucket(q)], p - 1);
    atomicAdd(&s.hist[bucket(len - (p - 1) * q)], 1);
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
  each([&](int b, int r, int tile, const TileKeys& k, int q, int p) {
    const int len = max(k.k1 - k.k0, 0);
    int slot = -1;
    if (p > 1) {
      slot = atomicAdd(&s.slots, p);
      const int e = atomicAdd(&s.n_splits, 1);
      if (slot + p <= a.max_slots && e < a.max_splits)
        a.splits[e] = ChunkSplit{b, tile, slot, p, s.row0[r], s.n[r], s.L[r], 0};
      else   // (cu that divides the rows cannot need more than the workspace holds)
        slot = INT_MIN;
    }
    for (int i = 0; i < p; ++i) {
      const bool whole = slot == INT_MIN && i == 0;   // (then the other pieces are empty)
      const int k0 = k.k0 + i * q, k1 = whole || i == p - 1 ? k.k1 : k0 + q;
      const int at = atomicAdd(&s.hist[bucket(i == p - 1 ? len - i * q : q)], 1);
      if (at >= a.max_units) continue;
      if (slot == INT_MIN && !whole) a.units[at] = ChunkUnit{b, 0, 0, 0, -1, 0, 0, 0};
      else a.units[at] = ChunkUnit{b, tile, k0, k1, slot < 0 ? -1 : slot + i, s.row0[r], s.n[r], s.L[r]};
    }
  });
  __syncthreads();
  if (tid == 0) {
    a.status[0] = s.bits;
    a.status[2] = min(s.n_splits, a.max_splits);
  }
}

// ------------------------------------------------------------------------------ merge

constexpr int MG_THREADS = 256;

// o = sum_i O_i 2^(m_i - m*) / sum_i l_i 2^(m_i - m*) over the pieces in key order; a thread takes four dims of a row.
template <class T, int D>
__global__ void __launch_bounds__(MG_THREADS) chunk_merge(ChunkAttnArgs a, int blocks) {
  constexpr int PR = MG_THREADS * 4 / D;   // rows per workgroup
  constexpr int U = 4;
  const int g = a.Hq / a.Hkv;
  const int n = a.status[2] * a.Hkv * blocks;
  for (int w = blockIdx.x; w < n; w += gridDim.x) {
    const int e = w / (a.Hkv * blocks), h = w / blocks % a.Hkv;
    const ChunkSplit s = a.splits[e];
    const int rr = w % blocks * PR + threadIdx.x / (D / 4);   // row of the tile
    const int c = s.tile * a.tile_rows + rr;
    if (rr >= a.tile_rows || c >= s.n * g) continue;
    const int d = threadIdx.x % (D / 4) * 4;
    const size_t p0 = ((size_t)s.slot * a.Hkv + h) * a.tile_rows + rr, step = (size_t)a.Hkv * a.tile_rows;
    float m = -INFINITY;
    for (int i = 0; i < s.pieces; i += U) {
      float v[U];
#pragma unroll
      for (int x = 0; x < U; ++x) v[x] = a.part_ml[(p0 + min(i + x, s.pieces - 1) * step) * 2];
#pragma unroll
      for (int x = 0; x < U; ++x) m = fmaxf(m, v[x]);
    }
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < s.pieces; i += U) {
      float2 ml[U];
      f32x4 o[U];
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const size_t p = p0 + min(i + x, s.pieces - 1) * step;
        ml[x] = *reinterpret_cast<const float2*>(a.part_ml + p * 2);
        o[x] = *reinterpret_cast<const f32x4*>(a.part_o + p * D + d);
      }
#pragma unroll
      for (int x = 0; x < U; ++x) {
        if (i + x >= s.pieces) break;
        if (ml[x].x == -INFINITY && ml[x].y == 0.f) continue;   // a piece the row sees nothing of
        const float f = __builtin_amdgcn_exp2f(ml[x].x - m_use);
        l += ml[x].y * f;
        acc += o[x] * f;
      }
    }
    const int tok = c / g;
    const long long pos = (long long)s.L + tok;
    const long long lo = a.window > 0 ? pos - a.window + 1 : 0;
    const float inv = min(pos + 1, (long long)a.cap) > lo ? 1.f / l : 0.f;
    acc *= inv;
    T* dst = static_cast<T*>(a.o) + ((size_t)(s.row0 + tok) * a.Hq + h * g + (c - tok * g)) * D + d;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(dst) = acc;
    else *reinterpret_cast<bf16x4*>(dst) = bf16x4{f2bf(acc[0]), f2bf(acc[1]), f2bf(acc[2]), f2bf(acc[3])};
  }
}

// ----------------------------------------------------------------------------- launch

// Tile of the units: rows per wave are 32; one, two or four waves by the rows a request can have (n g), so that a
// workgroup of few rows is not mostly idle waves.  Tiles of 32 keys where one wave or fp32 rows would make 64 too large.
template <class F>
auto with_variant(const ChunkAttnArgs& a, F f) {
  const long long R = (long long)a.max_new * (a.Hq / a.Hkv);
  auto by_rows = [&](auto t, auto d) {
    typedef typename decltype(t)::type T;
    constexpr int D = decltype(d)::value;
    constexpr int KT = sizeof(T) == 4 ? 32 : 64;
    if (R <= 32) return f(t, d, Int<1>{}, Int<32>{});
    if (R <= 64) return f(t, d, Int<2>{}, Int<KT>{});
    return f(t, d, Int<4>{}, Int<KT>{});
  };
  if (a.f32) return a.D == 128 ? by_rows(std::common_type<float>{}, Int<128>{}) : by_rows(std::common_type<float>{}, Int<64>{});
  return a.D == 128 ? by_rows(std::common_type<bf16>{}, Int<128>{}) : by_rows(std::common_type<bf16>{}, Int<64>{});
}

constexpr int CHUNK_TARGET = 1024;    // units (x KV heads) that splitting aims for
constexpr int CHUNK_MIN_SPLIT = 256;  // keys a piece has at least

}  // namespace

void chunk_bounds(ChunkAttnArgs& a) {
  with_variant(a, [&](auto, auto, auto nw, auto kt) {
    a.tile_rows = 32 * decltype(nw)::value;
    a.key_tile = decltype(kt)::value;
    return 0;
  });
  a.min_split = CHUNK_MIN_SPLIT;
  a.target = CHUNK_TARGET;
  const long long g = a.Hq / a.Hkv;
  const long long per_req = ((long long)a.max_new * g + a.tile_rows - 1) / a.tile_rows;
  const long long tiles = std::min((long long)a.T * g / a.tile_rows + a.B, per_req * a.B);
  // pieces of a tile, and of all tiles: see chunk_plan
  const long long len = (long long)a.cap + a.key_tile;
  const long long cuts = len > a.min_split ? (len + a.min_split - 1) / a.min_split : 1;
  const long long extra = (a.target + a.Hkv - 1) / a.Hkv;
  a.max_units = (int)std::min(tiles * cuts, tiles + extra);
  a.max_slots = cuts > 1 ? (int)std::min(tiles * cuts, 2 * extra) : 0;
  a.max_splits = (int)std::min(tiles, (long long)a.max_slots / 2);
}

hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(chunk_plan, dim3(1), dim3(PL_THREADS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  return with_variant(a, [&](auto t, auto d, auto nw, auto kt) -> hipError_t {
    typedef typename decltype(t)::type T;
    constexpr int D = decltype(d)::value, NW = decltype(nw)::value, KT = decltype(kt)::value;
    constexpr auto kern = chunk_attn_kernel<T, D, NW, KT>;
    static int slots_of[64] = {};   // resident workgroups, per device
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    int& slots = slots_of[dev & 63];
    if (slots == 0) {
      int cus = 0, per_cu = 0;
      hipError_t e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
      if (e == hipSuccess) e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kern, 64 * NW, 0);
      if (e != hipSuccess) return e;
      slots = cus * (per_cu > 0 ? per_cu : 1);
    }
    const long long items = (long long)a.max_units * a.Hkv;
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min(items, (long long)slots)), dim3(64 * NW), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.max_splits > 0) {
      const int blocks = (a.tile_rows * D / 4 + MG_THREADS - 1) / MG_THREADS;
      const long long wgs = (long long)a.max_splits * a.Hkv * blocks;
      hipLaunchKernelGGL((chunk_merge<T, D>), dim3((unsigned)std::min(wgs, 4096LL)), dim3(MG_THREADS), 0, s, a, blocks);
    }
    return hipGetLastError();
  });
}

}  // namespace hspec
