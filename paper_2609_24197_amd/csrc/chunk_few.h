// Units of attention over the 4-bit cache for requests of few rows (a token each, the last token and its drafts, a
// drafted block), where reading the cache is what counts.
//
// A wave owns NCT x 16 rows (token, query head of the group) as columns and walks the unit's keys by itself, 64 at a time:
//   S^T [keys x rows] = K Q^T   and   O^T [D x rows] += V^T P^T,   16 x 16 x 32 products.
// Lane l holds channels [D/4 c, D/4 (c + 1)), c = l / 16, of key l % 16 of every 16: of K that is the product's operand as
// it is, widened in registers (the channels are summed over, so any order of them serves, if Q has the same).  V^T wants
// its keys side by side: V goes, widened, through a piece of LDS of the wave's own, from which it is read transposed in the
// order in which S^T leaves a lane its keys.  No wave waits for another: there is no barrier in a unit.
#pragma once
#include "chunk_tile.h"

namespace hspec {
namespace {

template <int D_, int NCT_, int NW_>
struct Few {
  typedef bf16 T;
  static constexpr int D = D_, NCT = NCT_, NW = NW_;
  static constexpr int KT = NCT > 2 ? 32 : 64;   // keys of a step (what three blocks of rows leave registers for)
  static constexpr int NT = 64 * NW, ROWS = 16 * NCT * NW;
  static constexpr int WPE = NCT == 1 ? 3 : 2;   // waves per SIMD the registers are sized for
  static constexpr int STAGE = NW * 32 * D;   // elements of LDS: 32 keys of V of every wave
};

// Element offset of (key, channel d) in a wave's V: 16-byte piece p of a row lies at p ^ f, with f such that a
// transposing read's 8 rows of two pieces, and a write's 16 rows of one, fall into different banks.
template <int D>
__device__ __forceinline__ int few_off(int key, int d) {
  const int f = (D == 128 ? 2 * (key & 7) : key & 6) ^ ((key >> 3) & 1);
  return key * D + (((d >> 3) ^ f) << 3) + (d & 7);
}
// 4 keys (4 c + j, of the 16 from key0 on) x this lane's d of V^T.
template <int D>
__device__ __forceinline__ s16x4 few_v(const bf16* sV, int key0, int db, int lane) {
  const int key = key0 + 4 * (lane >> 4) + ((lane & 15) >> 2);
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(sV + few_off<D>(key, db * 16 + 4 * (lane & 3))));
}

template <bool ODD, class C>
__device__ __forceinline__ bool few_unit(const ChunkAttnArgs& a, const ChunkUnit& u, int h, bf16* stage) {
  constexpr int D = C::D, KT = C::KT, NCT = C::NCT;
  constexpr int CH = D / 4, NS = CH / 8, NB = D / 16, NK = KT / 16;   // channels of a lane, products per 16 keys, d blocks, groups of keys
  typedef typename std::conditional<D == 128, u32x4, uint2>::type Codes;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane >> 4, l16 = lane & 15;
  const int lps = 31 - __builtin_clz(a.ps);
  const int g = a.Hq / a.Hkv;
  const int R = u.n * g;
  const int c0 = u.tile * C::ROWS + wave * 16 * NCT;   // first row of this wave
  if (c0 >= R) return false;
  bf16* sV = stage + wave * 32 * D;
  const int back = a.window > 0 ? a.window - 1 : INT_MAX;
  auto sees_from = [&](int tok) { return max(u.L + tok - back, 0); };
  auto sees_to = [&](int tok) { return min(min(u.L + (a.block ? u.n : tok + 1), a.cap), u.k1); };
  const int t_first = c0 / g, t_last = min(c0 + 16 * NCT - 1, R - 1) / g;
  const int any_lo = sees_from(t_first), any_hi = sees_to(t_last), all_lo = sees_from(t_last), all_hi = sees_to(t_first);
  const int k_min = max(u.k0, any_lo);   // the first key that a row of this wave sees: those before it are not read
  const int held = a.k_new ? min(u.L, u.k1) : u.k1;

  // this lane's column of each 16: its token, its first element, the keys it sees
  int lo[NCT], hi[NCT];
  size_t at_q[NCT];
  bool real[NCT];
  bf16x8 qf[NCT][NS];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) {
    const int r = c0 + 16 * ct + l16;
    real[ct] = r < R;
    const int tok = real[ct] ? r / g : u.n - 1, hq = h * g + (real[ct] ? r - tok * g : 0);
    at_q[ct] = ((size_t)(u.row0 + tok) * a.Hq + hq) * D;
    lo[ct] = sees_from(tok);
    hi[ct] = real[ct] ? sees_to(tok) : 0;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      qf[ct][s] = real[ct] ? ld8(static_cast<const bf16*>(a.q) + at_q[ct] + CH * c + 8 * s) : zero8();
  }
  auto live = [&](int ct) { return ct == 0 || c0 + 16 * ct < R; };   // (uniform)

  // Ids of pages [pg0, pg0 + 64) and the 64 behind them, lane by lane; a step's pages lie in one such window, since its
  // keys and pg0 are aligned to steps.
  const int32_t* ptab = a.page_table + (size_t)u.b * a.max_pages;
  const int pg_end = held > k_min ? ((held - 1) >> lps) + 1 : 0;
  const int from = k_min / KT * KT;   // (u.k0 is a multiple of 64 too, and 16 keys lie in one page)
  int pg0 = (from >> lps) & ~3;
  auto ids_at = [&](int pg) { return pg + lane < pg_end ? ptab[pg + lane] : -1; };
  int ids = ids_at(pg0), ids_next = ids_at(pg0 + 64);
  // KT keys on their way: where each 16 of them begin in a cache, and which of them this lane's key is
  struct Place {
    size_t off[NK];       // of the head's part of the page
    unsigned bytes[NK];   // 0: no such page
  };
  const unsigned head_bytes = (unsigned)mx_head_bytes(a.ps, D), page_bytes = head_bytes * (unsigned)a.Hkv;
  const size_t at_h = (size_t)h * head_bytes;
  auto place = [&](int base) {
    Place x;
    if ((base >> lps) >= pg0 + 64) {
      pg0 += 64;
      ids = ids_next;
      ids_next = ids_at(pg0 + 64);
    }
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      const int pg = (base + 16 * t) >> lps;
      const unsigned id = (unsigned)__builtin_amdgcn_readlane(ids, (pg - pg0) & 63);
      const bool good = id < (unsigned)a.num_pages;
      x.bytes[t] = good ? head_bytes : 0u;
      x.off[t] = at_h + (size_t)(good ? id : 0u) * page_bytes;
      if (!good && base + 16 * t < held && base + 16 * t + 16 > k_min && lane == 0) set_status(a.status, ST_BAD_PAGE);
    }
    return x;
  };
  struct Raw {
    Codes code[NK];
    unsigned scale[NK];
  };
  const unsigned at_code = l16 * (D / 2) + c * (CH / 2), at_scale = a.ps * (D / 2) + l16 * (D / MX_BLOCK) + c * CH / MX_BLOCK;
  auto load = [&](const void* cache, int base, const Place& at, Raw& x) {
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      // (a key that no row sees reads as zeros, by an offset past the buffer)
      const bool in = (unsigned)(base + 16 * t + l16 - k_min) < (unsigned)(held - k_min);
      const unsigned row0 = (unsigned)(base + 16 * t) & (unsigned)(a.ps - 1);
      const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(static_cast<const uint8_t*>(cache) + at.off[t]), 0,
                                                       at.bytes[t], BUFFER_FLAGS);
      if constexpr (D == 128) {
        x.code[t] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b128(r, in ? at_code : BUF_OOB, row0 * (D / 2), 0));
      } else {
        x.code[t] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b64(r, in ? at_code : BUF_OOB, row0 * (D / 2), 0));
      }
      x.scale[t] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, in ? at_scale : BUF_OOB, row0 * (D / MX_BLOCK), 0);
    }
  };
  auto word = [](const Codes& x, int s) -> unsigned { return reinterpret_cast<const unsigned*>(&x)[s]; };

  f32x4 o[NCT][NB];
  float m_run[NCT], l_run[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) {
#pragma unroll
    for (int db = 0; db < NB; ++db) o[ct][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[ct] = -INFINITY;
    l_run[ct] = 0.f;
  }
  f32x4 st[NCT][NK];
  // Softmax of the scores of keys [base, base + 64) below end, and their values' part of the output.
  // value(t, s): channels 8 s .. of this lane's of V of its key of the t-th 16.
  auto attend = [&](int base, int end, auto value) {
    const bool full = base + KT <= min(all_hi, end) && base >= all_lo;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      if (!live(ct)) continue;
      if (!full) {
        const int top = min(hi[ct], end);
        const unsigned span = (unsigned)max(top - lo[ct], 0);
#pragma unroll
        for (int t = 0; t < NK; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((unsigned)(base + 16 * t + 4 * c + i - lo[ct]) >= span) st[ct][t][i] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, st[ct][t][i]);
      mx = wave_max16x4(mx) * a.scale_log2;
      if (__any(mx > m_run[ct] + CHUNK_SLACK)) {
        // a row's own scores alone decide: rows that share the wave may see keys that it does not
        const float m_new = mx > m_run[ct] + CHUNK_SLACK ? mx : m_run[ct];
        const float alpha = __builtin_amdgcn_exp2f(m_run[ct] - (m_new == -INFINITY ? 0.f : m_new));
        l_run[ct] *= alpha;
#pragma unroll
        for (int db = 0; db < NB; ++db) o[ct][db] *= alpha;
        m_run[ct] = m_new;
      }
      const float m_use = m_run[ct] == -INFINITY ? 0.f : m_run[ct];
#pragma unroll
      for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[ct][t][i], a.scale_log2, -m_use));
          st[ct][t][i] = e;
          l_run[ct] += e;
        }
    }
    // P enters as bf16: half a step is 2^-8 of each weight, as large as the output's own rounding; the sum above takes
    // the unrounded weights
#pragma unroll
    for (int t = 0; t < NK; t += 2) {
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int s = 0; s < NS; ++s)
          *reinterpret_cast<bf16x8*>(sV + few_off<D>(16 * t2 + l16, CH * c + 8 * s)) = value(t + t2, s);
      bf16x8 pf[NCT];
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[ct][j] = f2bf(st[ct][t + j / 4][j % 4]);
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        const s16x4 v0 = few_v<D>(sV, 0, db, lane), v1 = few_v<D>(sV, 16, db, lane);
        bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        if constexpr (ODD) {
          // values that are not finite are kept out of the product, where 0 x them would reach rows that do not see
          // them, and added to the rows that do, as sums that overflow (a NaN as +inf and -inf)
          s16x8 bits = __builtin_bit_cast(s16x8, vf), up, dn;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool fin = (bits[j] & 0x7f80) != 0x7f80, nan = !fin && (bits[j] & 0x7f);
            up[j] = (short)(!fin && (nan || bits[j] >= 0) ? 0x7f7f : 0);   // the largest bf16
            dn[j] = (short)(!fin && (nan || bits[j] < 0) ? 0xff7f : 0);
            if (!fin) bits[j] = 0;
          }
          vf = __builtin_bit_cast(bf16x8, bits);
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) {
            s16x8 sees;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int key = base + 16 * (t + j / 4) + 4 * c + j % 4;
              sees[j] = (short)(key >= lo[ct] && key < min(hi[ct], end) ? 0x7f7f : 0);
            }
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            o[ct][db] += mma16(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, sees), zero);
            o[ct][db] += mma16(__builtin_bit_cast(bf16x8, dn), __builtin_bit_cast(bf16x8, sees), zero);
          }
        }
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
          if (live(ct)) o[ct][db] = mma16(vf, pf[ct], o[ct][db]);
      }
    }
  };

  // cached keys: the next step's K is on its way from where this one's is multiplied, its V from where this one's has
  // gone into LDS
  if (from < held) {
    Raw rk, rv;
    Place at = place(from);
    load(a.k_cache, from, at, rk);
    load(a.v_cache, from, at, rv);
    for (int base = from; base < held; base += KT) {
      const bool more = base + KT < held;
#pragma unroll
      for (int t = 0; t < NK; ++t) {
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) st[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const bf16x8 kf = mx_widen(word(rk.code[t], s), rk.scale[t]);
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct)
            if (live(ct)) st[ct][t] = mma16(kf, qf[ct][s], st[ct][t]);
        }
      }
      if (more) {
        at = place(base + KT);
        load(a.k_cache, base + KT, at, rk);
      }
      attend(base, held, [&](int t, int s) { return mx_widen(word(rv.code[t], s), rv.scale[t]); });
      if (more) load(a.v_cache, base + KT, at, rv);
    }
  }
  // the new tokens' keys beside the cache, as they are
  if (a.k_new && u.k1 > u.L) {
    const int first = max(k_min, u.L);
    const size_t stride = (size_t)a.Hkv * D, at_new = (size_t)u.row0 * stride + h * D + CH * c;
    for (int base = first; base < any_hi; base += KT) {
      auto row = [&](const void* p, int t, int s) -> bf16x8 {
        const int key = base + 16 * t + l16;
        return key < u.k1 ? ld8(static_cast<const bf16*>(p) + at_new + (size_t)(key - u.L) * stride + 8 * s) : zero8();
      };
#pragma unroll
      for (int t = 0; t < NK; ++t) {
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) st[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const bf16x8 kf = row(a.k_new, t, s);
#pragma unroll
          for (int ct = 0; ct < NCT; ++ct) st[ct][t] = mma16(kf, qf[ct][s], st[ct][t]);
        }
      }
      attend(base, INT_MAX, [&](int t, int s) { return row(a.v_new, t, s); });
    }
  }

  // lane holds O[row l16][d = 16 db + 4 c + i]
  bool bad = false;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) {
    if (!live(ct)) continue;
    const float l = wave_sum16x4(l_run[ct]);
    if constexpr (!ODD) {
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= real[ct] && !(fabsf(o[ct][db][i]) < INFINITY);
    }
    if (!real[ct]) continue;
    if (u.slot < 0) {
      const float inv = hi[ct] > lo[ct] ? 1.f / l : 0.f;   // (a row that sees no key is zero)
      bf16* dst = static_cast<bf16*>(a.o) + at_q[ct] + 4 * c;
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        const f32x4 v = o[ct][db] * inv;
        *reinterpret_cast<bf16x4*>(dst + 16 * db) = bf16x4{f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
      }
    } else {
      const size_t pr = ((size_t)u.slot * a.Hkv + h) * C::ROWS + wave * 16 * NCT + 16 * ct + l16;
      float* po = a.part_o + pr * D + 4 * c;
#pragma unroll
      for (int db = 0; db < NB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db) = o[ct][db];
      if (c == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = float2{m_run[ct], l};
    }
  }
  return bad;
}

// Workgroup (column, head) does the units of its column one after the other.  (256 threads: see chunk_attn_kernel)
template <class C>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(C::WPE))) few_kernel(ChunkAttnArgs a) {
  __shared__ __align__(16) bf16 stage[C::STAGE];
  const int h = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv;
  const int end = a.first[w + 1];
  for (int i = a.first[w]; i < end; ++i) {
    const ChunkUnit u = a.units[i];
    const bool bad = few_unit<false, C>(a, u, h, stage);
    // (one entry a wave at most: the same item twice is done twice, with the same result)
    if (a.redo && __any(bad) && (threadIdx.x & 63) == 0) {
      const int at = atomicAdd(a.status + 3, 1);
      if (at < a.max_redo) a.redo[at] = i * a.Hkv + h;
    }
  }
}
// The units some row of which came out infinite or NaN, once more with masked values kept apart.
template <class C>
__global__ void __launch_bounds__(C::NT) few_redo_kernel(ChunkAttnArgs a) {
  __shared__ __align__(16) bf16 stage[C::STAGE];
  const int n = min(a.status[3], a.max_redo);
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int item = a.redo[i];
    const ChunkUnit u = a.units[item / a.Hkv];
    few_unit<true, C>(a, u, item % a.Hkv, stage);
  }
}

template <class C>
hipError_t launch_few(const ChunkAttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(few_kernel<C>, dim3((unsigned)a.columns * a.Hkv), dim3(C::NT), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.redo) {
    const unsigned items = (unsigned)std::min(256LL, (long long)a.max_units * a.Hkv);
    hipLaunchKernelGGL(few_redo_kernel<C>, dim3(items), dim3(C::NT), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return launch_merge<bf16, C::D>(a, s);
}

}  // namespace
}  // namespace hspec
