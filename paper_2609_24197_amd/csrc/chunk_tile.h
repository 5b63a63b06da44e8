// Kernels of attention over a paged cache, shared by the types of caches: units of a plan, merge of split rows.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "chunk_plan.h"
#include "common.h"
#include "mx.h"
#include "target.h"
#include "target_rows.h"

namespace hspec {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
#define LDS_AS __attribute__((address_space(3)))
#define GLB_AS __attribute__((address_space(1)))

constexpr int BUFFER_FLAGS = 0x00027000;   // 32-bit data, no swizzle

// Softmax reference maximum: raised, and O and the sum rescaled, only when a tile exceeds it by more than this
// many powers of two; probabilities then stay below 2^8.
constexpr float CHUNK_SLACK = 8.f;

// NW waves, KT keys per tile.  ONCE: a request's rows fit one tile, so its K and V are read once: non-temporal loads,
// and a die takes all heads of its units, so that it reads whole rows of the cache (64 requests of 17 tokens 256 us, 264
// the other way; of 1 token 212 either way); otherwise a die keeps to its KV heads, whose K and V the tiles of a
// request share in its L2 (three prompts 1325 us, 1440 the other way; 2000 tokens behind 30000 1905 and 1990).
// MX: the cache holds 4-bit values (mx.h); what a tile takes of it goes through registers, where it is widened to T.
template <class T_, int D_, int NW_, int KT_, bool ONCE_, bool MX_ = false>
struct Chunk {
  typedef T_ T;
  static constexpr bool MX = MX_;
  static constexpr int D = D_, NW = NW_, KT = KT_, AUX = ONCE_ ? 2 : 0;
  static constexpr bool ONCE = ONCE_;
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
  static constexpr int WPE = chunk_waves_per_simd(sizeof(T) == 4, D);   // waves per SIMD the registers are sized for
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

// The key of a lane of 16 that writes rows of kv_off's.
template <int CPR>
__device__ __forceinline__ int kv_lane(int l) {
  if constexpr (CPR == 16) return spread16<0, 2, 3, 1>(l);
  else if constexpr (CPR == 8) return spread16<1, 2, 3, 0>(l);
  else return l;
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

// One unit's rows of one KV head.  Returns whether this lane's row came out with a value that is not finite.
// ODD: a key that a row does not see has weight 0 in the second product, and where its V is infinite or NaN, 0 x V
// would reach the row all the same.  So in partly masked tiles such values are taken out of the product and added
// to the rows that see them, as sums that overflow (a NaN as +inf and -inf).
template <class C, bool ODD>
__device__ __forceinline__ bool chunk_unit(const ChunkAttnArgs& a, const ChunkUnit& u, int h, typename C::T* st0,
                                           typename C::T* st1) {
  typedef typename C::T T;
  constexpr int D = C::D, KT = C::KT;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NQ = F32 ? D / 8 : D / 16;        // 16-byte pieces of a row per lane
  typedef typename std::conditional<F32, f32x4, bf16x8>::type Frag;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, l32 = lane & 31;
  const int lps = 31 - __builtin_clz(a.ps);
  const int g = a.Hq / a.Hkv;
  const T* Kc = static_cast<const T*>(C::MX ? a.k_new : a.k_cache);
  const T* Vc = static_cast<const T*>(C::MX ? a.v_new : a.v_cache);
  const int row_elems = a.Hkv * D;
  const unsigned row_bytes = (unsigned)row_elems * (unsigned)sizeof(T);
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
  auto sees_to = [&](int tok) { return min(min(u.L + (C::MX && a.block ? u.n : tok + 1), a.cap), u.k1); };
  const int lo = sees_from(i_tok), hi0 = real ? sees_to(i_tok) : 0;
  const int any_lo = sees_from(t_first), any_hi0 = sees_to(t_last);
  const int all_lo = sees_from(t_last), all_hi0 = sees_to(t_first);
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

  // MX with the new tokens beside the cache: keys from `held` on are theirs, and a window may leave no cached one
  const int held = C::MX && a.k_new ? min(u.L, u.k1) : u.k1;
  const int ntiles = held > (C::MX ? k_min : u.k0) ? (held - u.k0 + KT - 1) / KT : 0;
  const int32_t* ptab = a.page_table + (size_t)u.b * a.max_pages;
  // Page ids [pg0, pg0 + 256) of the table, lane by lane in four registers (-1 past the unit's last page): a tile's
  // ids cost no load of their own, which would have to wait for the DMA that went out before it.
  int pg0 = 0, id0, id1, id2, id3;
  const int pg_end = held > u.k0 ? ((held - 1) >> lps) + 1 : 0;
  auto load_ids = [&](int pg) {
    pg0 = pg;
    const int e = pg + lane;
    id0 = e < pg_end ? ptab[e] : -1;
    id1 = e + 64 < pg_end ? ptab[e + 64] : -1;
    id2 = e + 128 < pg_end ? ptab[e + 128] : -1;
    id3 = e + 192 < pg_end ? ptab[e + 192] : -1;
  };
  load_ids(k_min >> lps);
  auto page_id = [&](int pg) -> int {
    const int e = pg - pg0;
    const int v0 = __builtin_amdgcn_readlane(id0, e & 63), v1 = __builtin_amdgcn_readlane(id1, e & 63);
    const int v2 = __builtin_amdgcn_readlane(id2, e & 63), v3 = __builtin_amdgcn_readlane(id3, e & 63);
    return e < 128 ? (e < 64 ? v0 : v1) : (e < 192 ? v2 : v3);
  };
  // this lane's row of DMA instruction i of a group, and the byte offset of its 16-byte piece from the group's first
  // row (the same in every group)
  auto dma_row = [&](int i) { return (i * 64 + lane) / C::CPR; };
  unsigned at[C::NI];
#pragma unroll
  for (int i = 0; i < C::NI; ++i) {
    const int r = wave * C::WROWS + dma_row(i);
    const int piece = kv_off<T, C::CPR>(r, (i * 64 + lane) % C::CPR * C::EPC) - r * D;   // stored at this lane's place
    at[i] = (unsigned)(dma_row(i) * row_elems + piece) * (unsigned)sizeof(T);
  }
  // DMA of the tile of keys [base, base + KT) into a stage: K rows, then V rows
  auto issue = [&](int base, T* sb) {
#pragma unroll
    for (int n = 0; n < C::NG; ++n) {
      const int r0 = wave * C::WROWS + n * C::GR;
      const int key0 = base + r0;
      const bool any = key0 + C::GR > k_min && key0 < u.k1;   // a group with nothing visible has no page
      int pid = -1;
      if constexpr (!C::MX) {
        if (any && (key0 >> lps) >= pg0 + 256) load_ids(key0 >> lps);
        pid = any ? page_id(key0 >> lps) : -1;
      }
      const bool good = C::MX ? any : (unsigned)pid < (unsigned)a.num_pages;
      // Buffers over the group's visible rows [first, last): what lies outside, a row before them by wrap-around, reads
      // as zeros without an access.  (No repeats of a row in its place: its infinity times weight 0 is NaN.)
      const int first = max(k_min - key0, 0), last = good ? min(u.k1 - key0, C::GR) : first;
      if (any && !good && lane == 0) set_status(a.status, ST_BAD_PAGE);
      const size_t row = C::MX ? (size_t)(good ? u.row0 + key0 + first - u.L : 0)
                               : ((size_t)(good ? pid : 0) << lps) + ((key0 + first) & (a.ps - 1));
      const size_t at0 = row * row_elems + h * D;
      const unsigned bytes = (unsigned)max(last - first, 0) * row_bytes, skip = (unsigned)first * row_bytes;
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(Kc + at0), 0, bytes, BUFFER_FLAGS);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(Vc + at0), 0, bytes, BUFFER_FLAGS);
      int to = r0 * D;
      asm volatile("" : "+s"(to));   // (else the LDS address of every instruction and stage takes a register of its own)
#pragma unroll
      for (int i = 0; i < C::NI; ++i) {
        T* dst = sb + to + i * 64 * C::EPC;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (LDS_AS void*)dst, 16, at[i] - skip, 0, 0, C::AUX);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (LDS_AS void*)(dst + C::TILE), 16, at[i] - skip, 0, 0, C::AUX);
      }
    }
  };

  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db) o[db] = zero16();
  float m_run = -INFINITY, l_run = 0.f;

  // the tile of keys [base, base + KT), of which MX takes those below end
  auto compute = [&](int base, int end, const T* sb) {
    const T* sK = sb;
    const T* sV = sb + C::TILE;
    const int any_hi = C::MX ? min(any_hi0, end) : any_hi0, all_hi = C::MX ? min(all_hi0, end) : all_hi0;
    const int hi = C::MX ? min(hi0, end) : hi0;
    const unsigned span = (unsigned)max(hi - lo, 0);
    if (!live || base >= any_hi || base + KT <= any_lo) return;   // (uniform) no key of the tile is visible here
    f32x16 st[C::NB];
#pragma unroll
    for (int kb = 0; kb < C::NB; ++kb) st[kb] = zero16();
    {
      // every K fragment first, then the products interleaved across key blocks
      Frag kf[C::NB][NQ];
#pragma unroll
      for (int s = 0; s < NQ; ++s)
#pragma unroll
        for (int kb = 0; kb < C::NB; ++kb)
          kf[kb][s] = *reinterpret_cast<const Frag*>(
              sK + kv_off<T, C::CPR>(kb * 32 + l32, F32 ? 8 * s + 4 * hf : 16 * s + 8 * hf));
#pragma unroll
      for (int s = 0; s < NQ; ++s)
#pragma unroll
        for (int kb = 0; kb < C::NB; ++kb) {
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              st[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[kb][s][e], qf[s][e], st[kb], 0, 0, 0);
          } else {
            st[kb] = mma32(kf[kb][s], qf[s], st[kb]);
          }
        }
    }

    const bool full = base + KT <= all_hi && base >= all_lo;
    if (!full) {
#pragma unroll
      for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = base + kb * 32 + 8 * (i / 4) + 4 * hf + i % 4;
          if ((unsigned)(key - lo) >= span) st[kb][i] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kb][i]);
    mx = half_max(mx) * a.scale_log2;
    if (__any(mx > m_run + CHUNK_SLACK)) {
      // a row's own scores alone decide: rows that share the wave may see keys that it does not
      const float m_new = mx > m_run + CHUNK_SLACK ? mx : m_run;
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

    // O^T += V^T P^T.  P enters as bf16 with bf16 storage (half a step is 2^-8 of each weight, and the output's own
    // rounding is as large); the sum above takes the unrounded weights.  This wave first while it has products to
    // issue: the other wave of the SIMD has its softmax to fill in (three prompts 1350 -> 1325 us, a chunk of 2000
    // tokens behind 30000 2008 -> 1905).
    __builtin_amdgcn_s_setprio(1);
    auto add_values = [&](auto masked_) {
      constexpr bool FIX = ODD && decltype(masked_)::value;
      if constexpr (F32) {
#pragma unroll
        for (int kb = 0; kb < C::NB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = kb * 32 + 8 * (i / 4) + 4 * hf + i % 4;
#pragma unroll
            for (int db = 0; db < C::NDB; ++db) {
              float v = sV[kv_off<T, C::CPR>(row, db * 32 + l32)];
              if constexpr (FIX) {
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
#pragma unroll
        for (int s = 0; s < 2 * C::NB; ++s) {
          bf16x8 pf;
#pragma unroll
          for (int j = 0; j < 8; ++j) pf[j] = f2bf(st[s / 2][8 * (s & 1) + j]);
#pragma unroll
          for (int db = 0; db < C::NDB; ++db) {
            bf16x8 vf = v_frag<C::CPR>(sV, s, db, lane);
            if constexpr (FIX) {
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
    if constexpr (ODD) {
      if (!full) add_values(std::true_type{});
      else add_values(std::false_type{});
    } else {
      add_values(std::false_type{});
    }
  };

  // `n` tiles from key `from` on, those of rows that are read as they are
  auto stream = [&](int from, int n) {
    if (n > 0) issue(from, st0);
    auto step = [&](int ti, T* mine, T* other) {
      wait_vmcnt<0>();
      wg_barrier();   // every wave's part of tile ti has landed, and every wave has left the other stage
      if (ti + 1 < n) issue(from + (ti + 1) * KT, other);
      compute(from + ti * KT, INT_MAX, mine);
      __builtin_amdgcn_s_setprio(0);
    };
    for (int t0 = 0; t0 < n; t0 += 2) {
      step(t0, st0, st1);
      if (t0 + 1 < n) step(t0 + 1, st1, st0);
    }
  };
  if constexpr (!C::MX) {
    stream(u.k0, ntiles);
  } else {
    // 4-bit tiles: tile t + 2 is on its way in registers while tile t + 1, widened, goes into the other stage and tile t is
    // multiplied.  A wave takes 16 keys of K or V at a time, a lane channels [CH c4, CH (c4 + 1)) of one key.  Loads go through
    // buffers, without branches: behind those the compiler would wait for every load under way.
    constexpr int CH = D / 4, G16 = KT / 16, NB = 2 * G16 / C::NW;
    static_assert(2 * G16 % C::NW == 0, "groups of 16 keys");
    typedef typename std::conditional<D == 128, u32x4, uint2>::type Codes;
    const int l16 = kv_lane<C::CPR>(lane & 15), c4 = lane >> 4;
    const unsigned head_bytes = (unsigned)mx_head_bytes(a.ps, D);
    const size_t page_bytes = mx_page_bytes(a.ps, D, a.Hkv);
    const size_t at_h = (size_t)h * head_bytes;
    const unsigned at_code = l16 * (D / 2) + c4 * (CH / 2), at_scale = a.ps * (D / 2) + l16 * (D / MX_BLOCK) + c4 * CH / MX_BLOCK;
    struct Raw {
      Codes code[NB];
      unsigned scale[NB];
    } raw;
    auto load = [&](int ti) {
      const int base = u.k0 + ti * KT;
      if ((base + KT - 1) >> lps >= pg0 + 256) load_ids(base >> lps);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int item = i * C::NW + wave, key0 = base + 16 * (item % G16);
        const bool any = key0 + 16 > k_min && key0 < held;   // (16 keys with nothing visible have no page)
        const int id = page_id(key0 >> lps);
        const bool good = any && (unsigned)id < (unsigned)a.num_pages;
        if (any && !good && lane == 0) set_status(a.status, ST_BAD_PAGE);
        const unsigned row0 = (unsigned)key0 & (unsigned)(a.ps - 1);
        // (a key that no row sees reads as zeros, by an offset past the buffer)
        const bool in = (unsigned)(key0 + l16 - k_min) < (unsigned)(held - k_min);
        const uint8_t* p = static_cast<const uint8_t*>(item < G16 ? a.k_cache : a.v_cache) + at_h + (size_t)(good ? id : 0) * page_bytes;
        const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, good ? head_bytes : 0u, BUFFER_FLAGS);
        if constexpr (D == 128) {
          raw.code[i] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b128(r, in ? at_code : BUF_OOB, row0 * (D / 2), 0));
        } else {
          raw.code[i] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b64(r, in ? at_code : BUF_OOB, row0 * (D / 2), 0));
        }
        raw.scale[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, in ? at_scale : BUF_OOB, row0 * (D / MX_BLOCK), 0);
      }
    };
    auto store = [&](T* sb) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int item = i * C::NW + wave, row = 16 * (item % G16) + l16;
        T* dst = sb + (item < G16 ? 0 : C::TILE);
#pragma unroll
        for (int w = 0; w < CH / 8; ++w) {
          const unsigned code = reinterpret_cast<const unsigned*>(&raw.code[i])[w];
          if constexpr (F32) {
            f32x4 lo4, hi4;
            mx_widen(code, raw.scale[i], lo4, hi4);
            *reinterpret_cast<f32x4*>(dst + kv_off<T, C::CPR>(row, CH * c4 + 8 * w)) = lo4;
            *reinterpret_cast<f32x4*>(dst + kv_off<T, C::CPR>(row, CH * c4 + 8 * w + 4)) = hi4;
          } else {
            *reinterpret_cast<bf16x8*>(dst + kv_off<T, C::CPR>(row, CH * c4 + 8 * w)) = mx_widen(code, raw.scale[i]);
          }
        }
      }
    };
    if (ntiles > 0) {
      load(0);
      store(st0);
      load(1);   // (keys past the last read as zeros)
    }
    auto step = [&](int ti, T* mine, T* other) {
      wait_vm_lgkm0<63>();
      wg_barrier();   // every wave's part of tile ti is in LDS, and every wave has left the other stage
      store(other);
      load(ti + 2);
      compute(u.k0 + ti * KT, held, mine);
      __builtin_amdgcn_s_setprio(0);
    };
    for (int t0 = 0; t0 < ntiles; t0 += 2) {
      step(t0, st0, st1);
      if (t0 + 1 < ntiles) step(t0 + 1, st1, st0);
    }
    wait_vm_lgkm0<63>();   // the last step has written a stage that nothing reads: done before the stages hold something else
    if (a.k_new) {
      const int from = max(u.k0, u.L);
      wg_barrier();   // (every wave has left both stages)
      stream(from, u.k1 > from ? (u.k1 - from + KT - 1) / KT : 0);
    }
  }

  // lane holds O[row l32][d = 32 db + 8 (i / 4) + 4 hf + i % 4]
  const float l = half_sum(l_run);
  bool bad = false;
  if constexpr (!ODD) {
#pragma unroll
    for (int db = 0; db < C::NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) bad |= !(fabsf(o[db][i]) < INFINITY);
  }
  if (!real) return false;
  if (u.slot < 0) {
    const float inv = hi0 > lo ? 1.f / l : 0.f;   // (a row that sees no key is zero)
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
  return bad;
}

template <class C>
// (256 threads for every NW: with fewer the compiler counts on one wave per SIMD and puts O into accumulation
// registers, which costs a copy of it both ways in every tile)
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(C::WPE)))
chunk_attn_kernel(ChunkAttnArgs a) {
  // one LDS object per stage, so that the compiler can tell the one being read from the one whose DMA is in flight
  __shared__ __align__(16) typename C::T st0[2 * C::TILE];
  __shared__ __align__(16) typename C::T st1[2 * C::TILE];
  __shared__ int s_item[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Work goes by class, one per die (workgroups go to the dies in turn): unit v of head h is in class v mod 8, or
  // (v Hkv + h) mod 8.  A workgroup's first ticket is its place in its class; the next come from the class's
  // counter, then from the other classes'.  Each claim goes out at the start of an item and is looked at at its end.
  const int grid = gridDim.x;   // a multiple of the classes
  const int cls = blockIdx.x % kChunkClasses, own = grid / kChunkClasses;
  auto place = [&](int c, int t) {   // item of a ticket
    return C::ONCE ? (t / a.Hkv * kChunkClasses + c) * a.Hkv + t % a.Hkv : t * kChunkClasses + c;
  };
  // the first item's unit, read beside the number of units (what it holds past them is not used)
  ChunkUnit u = a.units[min(place(cls, blockIdx.x / kChunkClasses) / a.Hkv, a.max_units - 1)];
  const int n_units = a.status[1];
  auto tickets = [&](int c) {   // of a class
    return C::ONCE ? (n_units - c + kChunkClasses - 1) / kChunkClasses * a.Hkv
                   : (n_units * a.Hkv - c + kChunkClasses - 1) / kChunkClasses;
  };
  const bool one_each = tickets(0) <= own;
  auto counter = [&](int c) { return a.queue + c * kChunkQueueStride; };
  auto item_of = [&](int c, int t) { return t < tickets(c) ? place(c, t) : -1; };
  // lanes of wave 0: an item of any class, or -1
  auto steal = [&]() -> int {
    for (;;) {
      int c = (cls + lane) % kChunkClasses, t = 0;
      if (lane < kChunkClasses) t = own + __hip_atomic_load(counter(c), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const unsigned long long some = __ballot(lane < kChunkClasses && t < tickets(c));
      if (!some) return -1;
      c = (cls + __builtin_ctzll(some)) % kChunkClasses;
      int got = 0;
      if (lane == 0) got = atomicAdd(counter(c), 1);
      const int it = item_of(c, own + __builtin_amdgcn_readfirstlane(got));
      if (it >= 0) return it;
    }
  };
  int turn = 0;
  auto shared = [&](int it) -> int {   // wave 0's item, for all
    if (tid == 0) s_item[turn] = it;
    __syncthreads();   // (and every wave is done with the last one)
    it = __builtin_amdgcn_readfirstlane(s_item[turn]);
    turn ^= 1;
    return it;
  };
  int item = item_of(cls, blockIdx.x / kChunkClasses);
  if (item < 0 && !one_each) {   // (uniform) fewer units in the class than workgroups
    item = shared(wave == 0 ? steal() : 0);
    u = a.units[max(item, 0) / a.Hkv];
  }
  while (item >= 0) {
    int ticket = 0;
    if (tid == 0 && !one_each) ticket = atomicAdd(counter(cls), 1);
    const int h = item % a.Hkv;
    const bool bad = chunk_unit<C, false>(a, u, h, st0, st1);
    // (one entry a wave at most: the same item twice is done twice, with the same result)
    if (a.redo && __any(bad) && lane == 0) {
      const int at = atomicAdd(a.status + 3, 1);
      if (at < a.max_redo) a.redo[at] = item;
    }
    if (one_each) break;
    int it = 0;
    if (wave == 0) {
      it = item_of(cls, own + __builtin_amdgcn_readfirstlane(ticket));
      if (it < 0) it = steal();
    }
    item = shared(it);
    u = a.units[max(item, 0) / a.Hkv];
  }
}

// The units some row of which came out infinite or NaN, once more with masked values kept apart (rare: the list is
// empty where V is finite and nothing overflows).
template <class C>
__global__ void __launch_bounds__(C::NT) chunk_redo_kernel(ChunkAttnArgs a) {
  __shared__ __align__(16) typename C::T st0[2 * C::TILE];
  __shared__ __align__(16) typename C::T st1[2 * C::TILE];
  const int n = min(a.status[3], a.max_redo);
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int item = a.redo[i];
    const ChunkUnit u = a.units[item / a.Hkv];
    chunk_unit<C, true>(a, u, item % a.Hkv, st0, st1);
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------ merge

constexpr int MG_THREADS = 256;

// o = sum_i O_i 2^(m_i - m*) / sum_i l_i 2^(m_i - m*) over a row's pieces, in an order of their own (not of time).
// Bound by the round trips of a row's loads: a workgroup takes one row, with its pieces spread over groups of D / 4
// threads, where that makes few workgroups (few rows, so perhaps many pieces each: 1 request of 32768 tokens, 64 pieces,
// 43 us for the whole call, 56 with a thread for all of a row's pieces), else 1024 / D rows (64 requests of
// 68 rows 256 us for the whole call, 291 with a row each).
constexpr int MG_FEW = 4096;   // workgroups up to which each takes one row

template <class T, int D>
__device__ __forceinline__ void merge_store(const ChunkAttnArgs& a, const ChunkSplit& s, int h, int c, int d, f32x4 acc, float l) {
  const int g = a.Hq / a.Hkv, tok = c / g;
  const long long pos = (long long)s.L + tok;
  const long long lo = a.window > 0 ? pos - a.window + 1 : 0;
  acc *= min(pos + 1, (long long)a.cap) > lo ? 1.f / l : 0.f;   // (a row that sees no key is zero)
  T* dst = static_cast<T*>(a.o) + ((size_t)(s.row0 + tok) * a.Hq + h * g + (c - tok * g)) * D + d;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(dst) = acc;
  else *reinterpret_cast<bf16x4*>(dst) = bf16x4{f2bf(acc[0]), f2bf(acc[1]), f2bf(acc[2]), f2bf(acc[3])};
}
// In columns, the last workgroup puts what the units' waves found into the status, which nothing else writes by then.
__device__ __forceinline__ bool merge_status(const ChunkAttnArgs& a, int waves) {   // whether this workgroup is that one
  if (!a.flags || blockIdx.x != gridDim.x - 1) return false;
  int bits = 0;
  for (int i = threadIdx.x; i < a.columns * a.Hkv * waves; i += MG_THREADS) bits |= a.flags[i];
  if (bits & 2) set_status(a.status, ST_BAD_PAGE);
  return true;
}
// (A piece that a row sees nothing of has m = -inf, l = 0 and O = 0; no piece is left out for its weight, so that a NaN
// among the scores or values of one shows as it does where a cache is not split.)
__device__ __forceinline__ float piece_weight(float m, float m_use) { return __builtin_amdgcn_exp2f(m - m_use); }

template <class T, int D>
__global__ void __launch_bounds__(MG_THREADS) chunk_merge_rows(ChunkAttnArgs a, int blocks, int waves) {
  if (merge_status(a, waves)) return;
  const int wgs = gridDim.x - (a.flags ? 1 : 0);
  constexpr int PR = MG_THREADS * 4 / D;   // rows per workgroup
  constexpr int U = 4;
  const int g = a.Hq / a.Hkv;
  const int n = a.status[2] * a.Hkv * blocks;
  for (int w = blockIdx.x; w < n; w += wgs) {
    const int e = w / (a.Hkv * blocks), h = w / blocks % a.Hkv;
    const ChunkSplit s = a.splits[e];
    const int rr = w % blocks * PR + threadIdx.x / (D / 4);   // row of the tile
    const int c = s.tile * a.tile_rows + rr;
    if (s.pieces < 2 || rr >= a.tile_rows || c >= s.n * g) continue;
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
        if (i + x >= s.pieces) continue;
        const float f = piece_weight(ml[x].x, m_use);
        l += ml[x].y * f;
        acc += o[x] * f;
      }
    }
    merge_store<T, D>(a, s, h, c, d, acc, l);
  }
}

template <class T, int D>
__global__ void __launch_bounds__(MG_THREADS) chunk_merge_row(ChunkAttnArgs a, int rows, int waves) {
  if (merge_status(a, waves)) return;
  const int wgs = gridDim.x - (a.flags ? 1 : 0);
  constexpr int TPR = D / 4, G = MG_THREADS / TPR;   // threads of a row, groups of pieces
  constexpr int U = 4, CH = MG_THREADS;              // pieces in flight per group, pieces per round
  __shared__ float s_w[CH], s_m[MG_THREADS / 64], s_l[MG_THREADS / 64];
  __shared__ __align__(16) f32x4 s_o[MG_THREADS];
  const int g = a.Hq / a.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.status[2] * a.Hkv * rows;
  for (int w = blockIdx.x; w < n; w += wgs) {
    const int e = w / (a.Hkv * rows), h = w / rows % a.Hkv, rr = w % rows;
    const ChunkSplit s = a.splits[e];
    const int c = s.tile * a.tile_rows + rr;
    if (s.pieces < 2 || c >= s.n * g) continue;   // (uniform)
    const size_t p0 = ((size_t)s.slot * a.Hkv + h) * a.tile_rows + rr, step = (size_t)a.Hkv * a.tile_rows;
    const int grp = tid / TPR, d = tid % TPR * 4;
    auto piece_o = [&](int i) { return *reinterpret_cast<const f32x4*>(a.part_o + (p0 + min(i, s.pieces - 1) * step) * D + d); };
    f32x4 o[U];   // the first pieces' O on its way beside the maxima
#pragma unroll
    for (int x = 0; x < U; ++x) o[x] = piece_o(grp + x * G);
    float m = -INFINITY;
    for (int i = tid; i < s.pieces; i += CH) m = fmaxf(m, a.part_ml[(p0 + i * step) * 2]);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < s.pieces; c0 += CH) {
      if (c0) __syncthreads();   // the last round's weights are read
      float f = 0.f;
      if (c0 + tid < s.pieces) {
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (p0 + (c0 + tid) * step) * 2);
        f = piece_weight(ml.x, m_use);
        l += ml.y * f;
      }
      s_w[tid] = f;
      __syncthreads();
      const int top = min(CH, s.pieces - c0);
      for (int i = grp; i < top; i += U * G) {
        if (c0 || i != grp) {
#pragma unroll
          for (int x = 0; x < U; ++x) o[x] = piece_o(c0 + i + x * G);
        }
#pragma unroll
        for (int x = 0; x < U; ++x) {
          if (i + x * G < top) acc += o[x] * s_w[i + x * G];
        }
      }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x);
    if (lane == 0) s_l[wave] = l;
    s_o[tid] = acc;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int x = 1; x < G; ++x) acc += s_o[x * TPR + tid];
      merge_store<T, D>(a, s, h, c, d, acc, (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]));
    }
    __syncthreads();   // s_m, s_l and s_o are filled again
  }
}

// ----------------------------------------------------------------------------- launch

template <class T, int D>
hipError_t launch_merge(const ChunkAttnArgs& a, hipStream_t s, int waves = 0) {
  const unsigned more = a.flags ? 1 : 0;   // the workgroup of merge_status
  if (a.max_splits > 0 || a.flags) {
    const long long rows = std::min((long long)a.tile_rows, (long long)a.max_new * (a.Hq / a.Hkv));
    const long long singles = (long long)a.max_splits * a.Hkv * rows;
    if (singles <= MG_FEW) {
      hipLaunchKernelGGL((chunk_merge_row<T, D>), dim3((unsigned)singles + more), dim3(MG_THREADS), 0, s, a, (int)rows, waves);
    } else {
      const int blocks = (int)((rows * D / 4 + MG_THREADS - 1) / MG_THREADS);
      const long long wgs = std::min((long long)a.max_splits * a.Hkv * blocks, 2048LL);
      hipLaunchKernelGGL((chunk_merge_rows<T, D>), dim3((unsigned)wgs + more), dim3(MG_THREADS), 0, s, a, blocks, waves);
    }
  }
  return hipGetLastError();
}

// Launches behind the plan: the units, those of them that are done again, the merge.
template <class C>
hipError_t launch_units(const ChunkAttnArgs& a, hipStream_t s) {
  constexpr int D = C::D, NW = C::NW;
  constexpr auto kern = chunk_attn_kernel<C>;
  static std::atomic<int> slots_of[64];   // resident workgroups, per device
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  int slots = slots_of[dev & 63].load(std::memory_order_relaxed);
  if (slots == 0) {
    int cus = 0, per_cu = 0;
    hipError_t e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (e == hipSuccess) e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kern, 64 * NW, 0);
    if (e != hipSuccess) return e;
    slots = std::max(cus * per_cu / kChunkClasses, 1) * kChunkClasses;
    slots_of[dev & 63].store(slots, std::memory_order_relaxed);
  }
  const long long items = (a.max_units + kChunkClasses - 1LL) / kChunkClasses * kChunkClasses * a.Hkv;
  hipLaunchKernelGGL(kern, dim3((unsigned)std::min(items, (long long)slots)), dim3(64 * NW), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.redo) {
    hipLaunchKernelGGL((chunk_redo_kernel<C>), dim3((unsigned)std::min(items, 256LL)), dim3(64 * NW), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return launch_merge<typename C::T, D>(a, s);
}

}  // namespace
}  // namespace hspec
