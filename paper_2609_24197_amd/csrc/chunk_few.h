// Units of attention over the 4-bit cache for requests of few rows (a token each, the last token and its drafts, a
// drafted block), where reading the cache is what counts.
//
//   S^T [keys x rows] = K Q^T   and   O^T [D x rows] += V^T P^T,   16 x 16 x 32 products:
// a wave owns NCT x 16 rows (token, query head of the group) as columns.  Lane l holds channels [D/4 c, D/4 (c + 1)),
// c = l / 16, of key l % 16 of every 16 (the channels are summed over, so any order of them serves, if Q has the same); V^T
// is read transposed from LDS in the order in which S^T leaves a lane its keys.
//
// Bound by HBM where a request has a token (64 of them, 512..8192 cached, 32 and 8 heads of 128: 67 us, 4.8 TB/s), past 32 rows
// by a step's chain of LDS, products and softmax, with two waves a SIMD (the whole call, a block of 16: 135 to 147 us by the card,
// 17 tokens: 169 to 176; the matrix units are busy a quarter of the time).
//
// Up to 32 rows (Few) a wave walks its keys by itself: K is the product's operand as it was loaded, widened in
// registers, V goes through a piece of LDS of the wave's own, and there is no barrier in a unit.  Past that (Share)
// the waves of a workgroup share what they widen: RW of them divide the rows, KW the keys of a step, and the KW results
// are put together at the unit's end.
#pragma once
#include "chunk_columns.h"
#include "chunk_tile.h"

namespace hspec {
namespace {

// Bits of what a unit found: a row that came out infinite or NaN, a page outside the pool.
enum : int { UNIT_ODD = 1, UNIT_BAD_PAGE = 2 };

// Element offset of (key, channel d) in LDS: 16-byte piece p of a row lies at p ^ f, with f such that a transposing
// read's 8 rows of two pieces, a fragment's 16 rows of one, and a write's fall into different banks.
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

// An fp32 value as the sum of three bf16, by cutting off bits: 8 + 8 + 8 of its 24, so that nothing is lost but what lies
// below 2^-133, bf16's smallest step.  (What is not finite is the first of them.)
struct Planes {
  unsigned bits[3];   // bf16 in the upper half
};
__device__ __forceinline__ Planes planes(float v) {
  Planes p;
  const bool fin = fabsf(v) < INFINITY;
  p.bits[0] = v == v ? __float_as_uint(v) & 0xffff0000u : 0x7fc00000u;
  const float r = fin ? v - __uint_as_float(p.bits[0]) : 0.f;
  p.bits[1] = __float_as_uint(r) & 0xffff0000u;
  p.bits[2] = __float_as_uint(r - __uint_as_float(p.bits[1]));
  return p;
}
// Of 8 of them, the PL-th bf16 of each (PL = 1: bf16 as it is).
template <int PL>
__device__ __forceinline__ void split8(const float* v, bf16x8 (&f)[PL]) {
  u32x4 w[PL];
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const Planes a = planes(v[j]), b = planes(v[j + 1]);
#pragma unroll
    for (int i = 0; i < PL; ++i) w[i][j / 2] = __builtin_amdgcn_perm(b.bits[i], a.bits[i], 0x07060302);
  }
#pragma unroll
  for (int i = 0; i < PL; ++i) f[i] = __builtin_bit_cast(bf16x8, w[i]);
}
// 8 values from memory as operands of products, or zeros.
template <class T, int PL>
__device__ __forceinline__ void operands(const void* p, size_t at, bool in, bf16x8 (&f)[PL]) {
  if constexpr (sizeof(T) == 2) {
    f[0] = in ? ld8(static_cast<const bf16*>(p) + at) : zero8();
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (in) {
      *reinterpret_cast<f32x4*>(v) = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
      *reinterpret_cast<f32x4*>(v + 4) = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at + 4);
    }
    split8<PL>(v, f);
  }
}

// A wave's rows: what they see, Q, and the softmax's running maximum, sum and output.  With fp32 rows Q and the weights
// enter as three bf16 each: the 4-bit values are bf16 exactly, so three products with 32-bit sums lose no more than one in 32
// bits does, at a fifth of its time.
template <class T, int D, int NCT, bool ODD>
struct FewRows {
  static constexpr int PL = sizeof(T) == 4 ? 3 : 1;
  static constexpr int CH = D / 4, NS = CH / 8, NB = D / 16;   // channels of a lane, products per 16 keys, d blocks
  int lo[NCT], hi[NCT];       // keys that this lane's column of each 16 sees
  int any_lo, any_hi, all_lo, all_hi;   // keys that any and that all rows of the wave see
  size_t at_q[NCT];
  bool real[NCT];
  bf16x8 qf[NCT][NS][PL];
  f32x4 o[NCT][NB];
  float m_run[NCT], l_run[NCT];
  int c0, R, lane, c;

  // (Columns past the last row go through all of it as zeros: branches around them would keep loads from running ahead.)

  __device__ __forceinline__ void init(const ChunkAttnArgs& a, const ChunkUnit& u, int h, int c0_) {
    const int g = a.Hq / a.Hkv, back = a.window > 0 ? a.window - 1 : INT_MAX;
    lane = threadIdx.x & 63;
    c = lane >> 4;
    c0 = c0_;
    R = u.n * g;
    auto sees_from = [&](int tok) { return max(u.L + tok - back, 0); };
    auto sees_to = [&](int tok) { return min(min(u.L + (a.block ? u.n : tok + 1), a.cap), u.k1); };
    const int t_first = min(c0, R - 1) / g, t_last = min(c0 + 16 * NCT - 1, R - 1) / g;
    any_lo = sees_from(t_first), any_hi = sees_to(t_last), all_lo = sees_from(t_last), all_hi = sees_to(t_first);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      const int r = c0 + 16 * ct + (lane & 15);
      real[ct] = r < R;
      const int tok = real[ct] ? r / g : u.n - 1, hq = h * g + (real[ct] ? r - tok * g : 0);
      at_q[ct] = ((size_t)(u.row0 + tok) * a.Hq + hq) * D;
      lo[ct] = sees_from(tok);
      hi[ct] = real[ct] ? sees_to(tok) : 0;
#pragma unroll
      for (int s = 0; s < NS; ++s)
        operands<T>(a.q, at_q[ct] + CH * c + 8 * s, real[ct], qf[ct][s]);
#pragma unroll
      for (int db = 0; db < NB; ++db) o[ct][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_run[ct] = -INFINITY;
      l_run[ct] = 0.f;
    }
  }

  // Softmax weights, in st, of the scores of keys [base, base + 16 NK) below end.
  template <int NK>
  __device__ __forceinline__ void weights(const ChunkAttnArgs& a, f32x4 (&st)[NCT][NK], int base, int end) {
    const bool full = base + 16 * NK <= min(all_hi, end) && base >= all_lo;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      if (!full) {
        const unsigned span = (unsigned)max(min(hi[ct], end) - lo[ct], 0);
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
  }

  // st[.][t] += scores of 16 keys, of which kf is the s-th 8 channels a lane.
  template <int NK>
  __device__ __forceinline__ void scores(f32x4 (&st)[NCT][NK], int t, int s, bf16x8 kf) const {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int i = 0; i < PL; ++i) st[ct][t] = mma16(kf, qf[ct][s][i], st[ct][t]);
  }

  // O += of the 32 keys from base on, whose weights are st[.][t] and st[.][t + 1] and whose V begins at sV.  With bf16
  // rows P enters as bf16: half a step is 2^-8 of each weight, as large as the output's own rounding; the sum takes the
  // unrounded weights.
  template <int NK>
  __device__ __forceinline__ void values(const f32x4 (&st)[NCT][NK], int t, const bf16* sV, int base, int end) {
    bf16x8 pf[NCT][PL];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      if constexpr (PL == 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[ct][0][j] = f2bf(st[ct][t + j / 4][j % 4]);
      } else {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = st[ct][t + j / 4][j % 4];
        split8<PL>(w, pf[ct]);
      }
    }
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
            const int key = base + 16 * (j / 4) + 4 * c + j % 4;
            sees[j] = (short)(key >= lo[ct] && key < min(hi[ct], end) ? 0x7f7f : 0);
          }
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          o[ct][db] += mma16(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, sees), zero);
          o[ct][db] += mma16(__builtin_bit_cast(bf16x8, dn), __builtin_bit_cast(bf16x8, sees), zero);
        }
      }
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int i = 0; i < PL; ++i) o[ct][db] = mma16(vf, pf[ct][i], o[ct][db]);
    }
  }

  // Lane holds O[row l16][d = 16 db + 4 c + i]: out, or as a partial result from row `part` of the unit's slot on.
  __device__ __forceinline__ int finish(const ChunkAttnArgs& a, const ChunkUnit& u, int h, int rows, int part) {
    bool bad = false;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
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
        T* dst = static_cast<T*>(a.o) + at_q[ct] + 4 * c;
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const f32x4 v = o[ct][db] * inv;
          if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(dst + 16 * db) = v;
          else *reinterpret_cast<bf16x4*>(dst + 16 * db) = bf16x4{f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
        }
      } else {
        const size_t pr = ((size_t)u.slot * a.Hkv + h) * rows + part + 16 * ct + (lane & 15);
        float* po = a.part_o + pr * D + 4 * c;
#pragma unroll
        for (int db = 0; db < NB; ++db) *reinterpret_cast<f32x4*>(po + 16 * db) = o[ct][db];
        if (c == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = float2{m_run[ct], l};
      }
    }
    return bad ? UNIT_ODD : 0;
  }
};

// Where keys lie.  Ids of pages [pg0, pg0 + 64) and the 64 behind them, lane by lane; a step's pages lie in one such
// window, since its keys and pg0 are aligned to 64 keys.
struct FewPages {
  const int32_t* tab;
  int pg0, end, ids, next, lps, num;

  __device__ __forceinline__ int at(int pg) const {
    const int e = pg + (int)(threadIdx.x & 63);
    return e < end ? tab[e] : -1;
  }
  __device__ __forceinline__ void init(const ChunkAttnArgs& a, int b, int from, int held) {
    lps = 31 - __builtin_clz(a.ps);
    num = a.num_pages;
    tab = a.page_table + (size_t)b * a.max_pages;
    end = held > from ? ((held - 1) >> lps) + 1 : 0;
    pg0 = (from >> lps) & ~3;
    ids = at(pg0);
    next = at(pg0 + 64);
  }
  __device__ __forceinline__ void step(int base) {   // before the pages of the 64 keys from base on are looked up
    if ((base >> lps) >= pg0 + 64) {
      pg0 += 64;
      ids = next;
      next = at(pg0 + 64);
    }
  }
  // id of the page of `key` (the same for the wave), or -1
  __device__ __forceinline__ int page(int key) const {
    const int id = __builtin_amdgcn_readlane(ids, ((key >> lps) - pg0) & 63);
    return (unsigned)id < (unsigned)num ? id : -1;
  }
};

// ---------------------------------------------------------------- a wave by itself

// (fp32 rows past 16 are divided over NW such waves, which have more to multiply than to widen.)
template <class T_, int D_, int NCT_, int NW_>
struct Few {
  typedef T_ T;
  static constexpr int D = D_, NCT = NCT_, NW = NW_;
  static constexpr int KT = 64, NT = 64 * NW, ROWS = 16 * NCT * NW;
  static constexpr int WPE = NCT == 1 && sizeof(T) == 2 ? 3 : 2;   // waves per SIMD the registers are sized for
  static constexpr int VK = NCT == 1 ? 32 : KT;                    // keys of V in LDS at a time
  static constexpr int LDS = NW * VK * D;                          // elements
  static constexpr int AUX = NW == 1 ? 2 : 0;                      // loads past the L2 where no other wave wants the keys
};

template <bool ODD, class C>
__device__ __forceinline__ int few_unit(C, const ChunkAttnArgs& a, const ChunkUnit& u, int h, bf16* lds) {
  typedef typename C::T T;
  constexpr int D = C::D, KT = C::KT, NCT = C::NCT, NK = KT / 16, VK = C::VK;
  typedef FewRows<T, D, NCT, ODD> Rows;
  constexpr int CH = Rows::CH, NS = Rows::NS, PL = Rows::PL;
  typedef typename std::conditional<D == 128, u32x4, uint2>::type Codes;
  const int lane = threadIdx.x & 63, c = lane >> 4, l16 = lane & 15;
  const int wave = C::NW > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, c0 = wave * 16 * NCT;
  if (c0 >= u.n * (a.Hq / a.Hkv)) return 0;
  bf16* sV = lds + wave * VK * D;
  const int held = a.k_new ? min(u.L, u.k1) : u.k1;
  Rows x;
  x.init(a, u, h, c0);
  const int k_min = max(u.k0, x.any_lo);   // the first key that a row sees: those before it are not read
  const int from = k_min / KT * KT;        // (u.k0 is a multiple of 64 too, so that 16 keys lie in one page)
  FewPages pages;
  pages.init(a, u.b, from, held);
  int found = 0;

  // KT keys on their way: where each 16 of them begin in a cache
  struct Place {
    size_t off[NK];       // of the head's part of the page
    unsigned bytes[NK];   // 0: no such page
  };
  const unsigned head_bytes = (unsigned)mx_head_bytes(a.ps, D);
  const size_t page_bytes = mx_page_bytes(a.ps, D, a.Hkv);
  const size_t at_h = (size_t)h * head_bytes;
  auto place = [&](int base) {
    Place p;
    pages.step(base);
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      const int id = pages.page(base + 16 * t);
      p.bytes[t] = id >= 0 ? head_bytes : 0u;
      p.off[t] = at_h + (size_t)max(id, 0) * page_bytes;
      if (id < 0 && base + 16 * t < held && base + 16 * t + 16 > k_min) found = UNIT_BAD_PAGE;
    }
    return p;
  };
  struct Raw {
    Codes code[NK];
    unsigned scale[NK];
  };
  // the key of 16 whose V this lane takes (16 bf16 rows wait for HBM, not for LDS, and have no register to spare: 74 us for 64
  // requests of a token with the lane's own key, 76 with this)
  constexpr bool OWN = NCT == 1 && sizeof(T) == 2;
  const int v16 = OWN ? l16 : D == 128 ? spread16<0, 1, 3, 2>(l16) : spread16<1, 2, 3, 0>(l16);
  const unsigned at_code = l16 * (D / 2) + c * (CH / 2), at_scale = a.ps * (D / 2) + l16 * (D / MX_BLOCK) + c * CH / MX_BLOCK;
  const unsigned at_code_v = v16 * (D / 2) + c * (CH / 2), at_scale_v = a.ps * (D / 2) + v16 * (D / MX_BLOCK) + c * CH / MX_BLOCK;
  auto load = [&](auto v, const void* cache, int base, const Place& p, Raw& w) {
    constexpr bool V = decltype(v)::value && !OWN;
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      // (a key that no row sees reads as zeros, by an offset past the buffer)
      const bool in = (unsigned)(base + 16 * t + (V ? v16 : l16) - k_min) < (unsigned)(held - k_min);
      const unsigned row0 = (unsigned)(base + 16 * t) & (unsigned)(a.ps - 1);
      const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(static_cast<const uint8_t*>(cache) + p.off[t]), 0,
                                                       p.bytes[t], BUFFER_FLAGS);
      if constexpr (D == 128) {
        w.code[t] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b128(r, in ? (V ? at_code_v : at_code) : BUF_OOB, row0 * (D / 2), C::AUX));
      } else {
        w.code[t] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b64(r, in ? (V ? at_code_v : at_code) : BUF_OOB, row0 * (D / 2), C::AUX));
      }
      w.scale[t] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, in ? (V ? at_scale_v : at_scale) : BUF_OOB, row0 * (D / MX_BLOCK), C::AUX);
    }
  };
  auto wide = [](const Raw& w, int t, int s) { return mx_widen(reinterpret_cast<const unsigned*>(&w.code[t])[s], w.scale[t]); };

  f32x4 st[NCT][NK];
  auto clear = [&]() {
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int t = 0; t < NK; ++t) st[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  // Groups [t0, t1) of V into LDS; value(t, s): channels 8 s .. of this lane's of its key (v16) of the t-th 16.
  auto put = [&](int t0, int t1, auto value) {
#pragma unroll
    for (int t = t0; t < t1; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s)
        *reinterpret_cast<bf16x8*>(sV + few_off<D>(16 * t % VK + (OWN ? l16 : v16), CH * c + 8 * s)) = value(t, s);
  };
  // (VK < KT: V goes into LDS here, 32 keys at a time)
  auto attend = [&](int base, int end, auto value) {
    x.weights(a, st, base, end);
#pragma unroll
    for (int t = 0; t < NK; t += 2) {
      if constexpr (VK < KT) put(t, t + 2, value);
      x.values(st, t, sV + 16 * t % VK * D, base + 16 * t, end);
    }
  };

  // cached keys, if a row sees one: the next step's are on their way from where this one's are multiplied (K) or have gone
  // into LDS (V)
  if (k_min < held) {
    Raw rk, rv;
    Place p = place(from);
    load(std::false_type{}, a.k_cache, from, p, rk);
    load(std::true_type{}, a.v_cache, from, p, rv);
    for (int base = from; base < held; base += KT) {
      auto value = [&](int t, int s) { return wide(rv, t, s); };
      p = place(base + KT);   // (keys past the last read as zeros; a branch around a load would have the next one wait for all)
      if constexpr (VK == KT) {
        put(0, NK, value);
        load(std::true_type{}, a.v_cache, base + KT, p, rv);
      }
      clear();
#pragma unroll
      for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int s = 0; s < NS; ++s) x.scores(st, t, s, wide(rk, t, s));
      load(std::false_type{}, a.k_cache, base + KT, p, rk);
      attend(base, held, value);
      if constexpr (VK < KT) load(std::true_type{}, a.v_cache, base + KT, p, rv);
    }
  }
  // the new tokens' keys beside the cache, as they are
  if (a.k_new && u.k1 > u.L) {
    const size_t stride = (size_t)a.Hkv * D, at_new = (size_t)u.row0 * stride + h * D + CH * c;
    for (int base = max(k_min, u.L); base < x.any_hi; base += KT) {
      auto row = [&](auto v, const void* p, int t, int s, bf16x8 (&f)[PL]) {
        const int key = base + 16 * t + (decltype(v)::value && !OWN ? v16 : l16);
        operands<T>(p, at_new + (size_t)(key - u.L) * stride + 8 * s, key < u.k1, f);
      };
      clear();
#pragma unroll
      for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          bf16x8 kf[PL];
          row(std::false_type{}, a.k_new, t, s, kf);
#pragma unroll
          for (int i = 0; i < PL; ++i) x.scores(st, t, s, kf[i]);
        }
      x.weights(a, st, base, INT_MAX);
#pragma unroll
      for (int t = 0; t < NK; t += 2)
#pragma unroll
        for (int i = 0; i < PL; ++i) {
          put(t, t + 2, [&](int t2, int s) {
            bf16x8 vf[PL];
            row(std::true_type{}, a.v_new, t2, s, vf);
            return vf[i];
          });
          x.values(st, t, sV + 16 * t % VK * D, base + 16 * t, INT_MAX);
        }
    }
  }
  return found | x.finish(a, u, h, C::ROWS, c0);
}

// ------------------------------------------------------------- waves share a step

// RW x KW waves: wave (r, k) has rows 32 r .. of the tile and keys 32 k .. of every KT, 32 x 32 x 16 products (as
// chunk_unit's, whose operands' layouts these are).
template <int D_, int RW_, int KW_>
struct Share {
  typedef bf16 T;
  static constexpr int D = D_, RW = RW_, KW = KW_;
  static constexpr int NW = RW * KW, KT = 64, NT = 64 * NW, ROWS = 32 * RW;
  static constexpr int WPE = 2;
  static constexpr int TILE = KT * D, CPR = D / 8;
  static constexpr int MERGE = KW > 1 ? ROWS * (D + 4) * 2 : 0;     // elements that results take on their way between waves
  static constexpr int LDS = 4 * TILE > MERGE ? 4 * TILE : MERGE;   // two stages of K and V
  static_assert(KW <= 2 && NW == 4, "waves");
};

template <bool ODD, class C>
__device__ __forceinline__ int share_unit(C, const ChunkAttnArgs& a, const ChunkUnit& u, int h, bf16* lds) {
  constexpr int D = C::D, KT = C::KT, TILE = C::TILE, CPR = C::CPR;
  constexpr int NQ = D / 16, NDB = D / 32, NKB = KT / 32 / C::KW;   // products per 32 keys, d blocks, 32-key blocks of a wave
  constexpr int CH = D / 4, NS = CH / 8;
  typedef typename std::conditional<D == 128, u32x4, uint2>::type Codes;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave / C::KW, kw = wave % C::KW;
  const int g = a.Hq / a.Hkv, R = u.n * g, c0 = rw * 32, c = c0 + l32;
  const bool live = c0 < R, real = c < R;
  const int tok = real ? c / g : u.n - 1, hq = h * g + (real ? c - tok * g : 0);
  const size_t at_q = ((size_t)(u.row0 + tok) * a.Hq + hq) * D;
  const int back = a.window > 0 ? a.window - 1 : INT_MAX;
  auto sees_from = [&](int t) { return max(u.L + t - back, 0); };
  auto sees_to = [&](int t) { return min(min(u.L + (a.block ? u.n : t + 1), a.cap), u.k1); };
  const int lo = sees_from(tok), hi0 = real ? sees_to(tok) : 0;
  const int t_first = min(c0, R - 1) / g, t_last = min(c0 + 31, R - 1) / g;
  const int any_lo = sees_from(t_first), any_hi0 = sees_to(t_last), all_lo = sees_from(t_last), all_hi0 = sees_to(t_first);
  const int k_min = max(u.k0, sees_from(0));   // the first key that a row of the unit sees
  const int cached = a.k_new ? min(u.L, u.k1) : u.k1, held = cached > k_min ? cached : 0;   // (0: no row sees a cached key)
  const int from = k_min / KT * KT;
  FewPages pages;
  pages.init(a, u.b, from, held);
  int found = 0;
  bf16x8 qf[NQ];
#pragma unroll
  for (int s = 0; s < NQ; ++s) qf[s] = real ? ld8(static_cast<const bf16*>(a.q) + at_q + 16 * s + 8 * hf) : zero8();
  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[db] = zero16();
  float m_run = -INFINITY, l_run = 0.f;

  // A wave takes 16 keys of K and of V a step, a lane channels [CH c4, CH (c4 + 1)) of one key.  Loads go through buffers,
  // without branches: behind those the compiler would wait for every load under way.
  const int l16 = kv_lane<CPR>(lane & 15), c4 = lane >> 4, k16 = 16 * wave;
  struct Raw {
    Codes code[2];   // K, V
    unsigned scale[2];
  };
  const unsigned head_bytes = (unsigned)mx_head_bytes(a.ps, D);
  const size_t page_bytes = mx_page_bytes(a.ps, D, a.Hkv);
  const size_t at_h = (size_t)h * head_bytes;
  const unsigned at_code = l16 * (D / 2) + c4 * (CH / 2), at_scale = a.ps * (D / 2) + l16 * (D / MX_BLOCK) + c4 * CH / MX_BLOCK;
  auto load = [&](int base, Raw& w) {
    pages.step(base);
    const int key0 = base + k16, id = pages.page(key0);
    if (id < 0 && key0 < held && key0 + 16 > k_min) found = UNIT_BAD_PAGE;
    const unsigned row0 = (unsigned)key0 & (unsigned)(a.ps - 1);
    const size_t off = at_h + (size_t)max(id, 0) * page_bytes;
    // (a key that no row sees reads as zeros, by an offset past the buffer)
    const bool in = (unsigned)(key0 + l16 - k_min) < (unsigned)(held - k_min);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* p = static_cast<const uint8_t*>(i ? a.v_cache : a.k_cache) + off;
      const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, id >= 0 ? head_bytes : 0u, BUFFER_FLAGS);
      if constexpr (D == 128) {
        w.code[i] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b128(r, in ? at_code : BUF_OOB, row0 * (D / 2), 2));
      } else {
        w.code[i] = __builtin_bit_cast(Codes, __builtin_amdgcn_raw_buffer_load_b64(r, in ? at_code : BUF_OOB, row0 * (D / 2), 2));
      }
      w.scale[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, in ? at_scale : BUF_OOB, row0 * (D / MX_BLOCK), 2);
    }
  };
  auto store = [&](const Raw& w, bf16* st) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int s = 0; s < NS; ++s)
        *reinterpret_cast<bf16x8*>(st + i * TILE + kv_off<bf16, CPR>(k16 + l16, CH * c4 + 8 * s)) =
            mx_widen(reinterpret_cast<const unsigned*>(&w.code[i])[s], w.scale[i]);
  };
  // keys [base, base + KT) below end of a stage
  auto compute = [&](int base, int end, const bf16* stage) {
    const int hi = min(hi0, end), all_hi = min(all_hi0, end), any_hi = min(any_hi0, end);
    const unsigned span = (unsigned)max(hi - lo, 0);
    const int key0 = 32 * NKB * kw, mine = base + key0;   // this wave's keys
    if (!live || mine >= any_hi || mine + 32 * NKB <= any_lo) return;   // (uniform)
    f32x16 st[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      bf16x8 kf[NQ];
#pragma unroll
      for (int s = 0; s < NQ; ++s) kf[s] = ld8(stage + kv_off<bf16, CPR>(key0 + 32 * kb + l32, 16 * s + 8 * hf));
      st[kb] = zero16();
#pragma unroll
      for (int s = 0; s < NQ; ++s) st[kb] = mma32(kf[s], qf[s], st[kb]);
    }
    // V is on its way from LDS beside the products and the softmax, 32 keys ahead (the scheduler would have each read right
    // before its use)
    bf16x8 vv[2][NDB];
    auto fetch = [&](int s) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) vv[s % 2][db] = v_frag<CPR>(stage + TILE, key0 / 16 + s, db, lane);
    };
    fetch(0);
    fetch(1);
    __builtin_amdgcn_sched_barrier(0);
    if (!(mine + 32 * NKB <= all_hi && mine >= all_lo)) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((unsigned)(mine + 32 * kb + 8 * (i / 4) + 4 * hf + i % 4 - lo) >= span) st[kb][i] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kb][i]);
    mx = half_max(mx) * a.scale_log2;
    if (__any(mx > m_run + CHUNK_SLACK)) {   // (a row's own scores alone decide)
      const float m_new = mx > m_run + CHUNK_SLACK ? mx : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        st[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][i], a.scale_log2, -m_use));
        l_run += st[kb][i];
      }
#pragma unroll
    for (int s = 0; s < 2 * NKB; ++s) {   // (P as bf16: see FewRows)
      bf16x8 pf;
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[j] = f2bf(st[s / 2][8 * (s & 1) + j]);
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        bf16x8 vf = vv[s % 2][db];
        if constexpr (ODD) {   // (see FewRows)
          s16x8 bits = __builtin_bit_cast(s16x8, vf), up, dn, sees;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool fin = (bits[j] & 0x7f80) != 0x7f80, nan = !fin && (bits[j] & 0x7f);
            const int key = mine + 16 * s + 8 * (j / 4) + 4 * hf + j % 4;
            up[j] = (short)(!fin && (nan || bits[j] >= 0) ? 0x7f7f : 0);
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
      if (s + 2 < 2 * NKB) fetch(s + 2);
    }
  };
  bf16 *st0 = lds, *st1 = lds + 2 * TILE;

  // cached keys: step t is multiplied while step t + 1 goes into the other stage and the two behind it are on their way
  // (keys past the last read as zeros)
  const int n = held > from ? (held - from + KT - 1) / KT : 0;
  if (n > 0) {
    Raw r0, r1;
    load(from, r0);
    load(from + KT, r1);
    wg_barrier();   // (the stages are free: another unit may have used them)
    store(r0, st0);
    load(from + 2 * KT, r0);
    auto step = [&](int t, bf16* mine, bf16* other, Raw& w) {
      wait_vm_lgkm0<63>();
      wg_barrier();   // every wave's part of step t is in LDS, and every wave has left the other stage
      store(w, other);
      load(from + (t + 3) * KT, w);
      compute(from + t * KT, held, mine);
    };
    for (int t = 0; t < n; t += 2) {
      step(t, st0, st1, r1);
      if (t + 1 < n) step(t + 1, st1, st0, r0);
    }
    // the last step has written a stage that nothing reads, and a wave without rows or visible keys comes straight from that:
    // a barrier waits for no write, and what lies behind the next one puts other things there
    wait_vm_lgkm0<63>();
  }
  // the new tokens' keys beside the cache, as they are
  if (a.k_new && u.k1 > u.L) {
    const size_t stride = (size_t)a.Hkv * D, at_new = (size_t)u.row0 * stride + h * D;
    for (int base = max(k_min, u.L); base < u.k1; base += KT) {
      wg_barrier();
      for (int i = tid; i < 2 * KT * D / 8; i += C::NT) {
        const bool is_k = i < KT * D / 8;
        const int row = i / (D / 8) % KT, d = i % (D / 8) * 8, key = base + row;
        const bf16* p = static_cast<const bf16*>(is_k ? a.k_new : a.v_new);
        *reinterpret_cast<bf16x8*>(st0 + (is_k ? 0 : TILE) + kv_off<bf16, CPR>(row, d)) =
            key < u.k1 ? ld8(p + at_new + (size_t)(key - u.L) * stride + d) : zero8();
      }
      wait_vm_lgkm0<63>();
      wg_barrier();
      compute(base, INT_MAX, st0);
    }
  }
  float l = half_sum(l_run);
  // the results of the two halves of the keys, put together by the first
  if constexpr (C::KW > 1) {
    wg_barrier();
    float* row = reinterpret_cast<float*>(lds) + (size_t)c * (D + 4);
    if (kw == 1) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(row + 32 * db + 8 * q + 4 * hf) =
              f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      if (hf == 0) *reinterpret_cast<float2*>(row + D) = float2{m_run, l};
    }
    wait_vm_lgkm0<63>();
    wg_barrier();
    if (kw == 0) {
      const float2 ml = *reinterpret_cast<const float2*>(row + D);
      const float m = fmaxf(m_run, ml.x), m_use = m == -INFINITY ? 0.f : m;
      const float f0 = __builtin_amdgcn_exp2f(m_run - m_use), f1 = __builtin_amdgcn_exp2f(ml.x - m_use);
      m_run = m;
      l = l * f0 + ml.y * f1;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 other = *reinterpret_cast<const f32x4*>(row + 32 * db + 8 * q + 4 * hf);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[db][4 * q + i] = o[db][4 * q + i] * f0 + other[i] * f1;
        }
    }
  }
  if (!real || kw != 0) return found;
  // lane holds O[row l32][d = 32 db + 8 q + 4 hf + i]
  bool bad = false;
  const float inv = hi0 > lo ? 1.f / l : 0.f;   // (a row that sees no key is zero)
  bf16* dst = static_cast<bf16*>(a.o) + at_q + 4 * hf;
  const size_t pr = ((size_t)max(u.slot, 0) * a.Hkv + h) * C::ROWS + c;
  float* po = a.part_o + pr * D + 4 * hf;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 v = {o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      if constexpr (!ODD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= !(fabsf(v[i]) < INFINITY);
      }
      if (u.slot < 0) {
        v *= inv;
        *reinterpret_cast<bf16x4*>(dst + 32 * db + 8 * q) = bf16x4{f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
      } else {
        *reinterpret_cast<f32x4*>(po + 32 * db + 8 * q) = v;
      }
    }
  if (u.slot >= 0 && hf == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = float2{m_run, l};
  return found | (bad ? UNIT_ODD : 0);
}

// ----------------------------------------------------------------------------- launch

template <bool ODD, class T, int D, int NCT, int NW>
__device__ __forceinline__ int run_unit(Few<T, D, NCT, NW> v, const ChunkAttnArgs& a, const ChunkUnit& u, int h, bf16* lds) {
  return few_unit<ODD>(v, a, u, h, lds);
}
template <bool ODD, int D, int RW, int KW>
__device__ __forceinline__ int run_unit(Share<D, RW, KW> v, const ChunkAttnArgs& a, const ChunkUnit& u, int h, bf16* lds) {
  return share_unit<ODD>(v, a, u, h, lds);
}

__device__ __forceinline__ ChunkUnit uniform(ChunkUnit u) {   // (the same in every lane, which the compiler cannot tell)
  auto f = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  return ChunkUnit{f(u.b), f(u.tile), f(u.k0), f(u.k1), f(u.slot), f(u.row0), f(u.n), f(u.L)};
}

// Units of a column: the plan's, or found here.  Every wave of the workgroup calls it.
struct ColumnUnits {
  const ChunkUnit* at;
  int n;
};
__device__ __forceinline__ ColumnUnits units_of(const ChunkAttnArgs& a, int w, ChunkUnit* found) {
  if (a.first) {
    const int i = a.first[w];
    return ColumnUnits{a.units + i, a.first[w + 1] - i};
  }
  const LanePlan p = lane_plan(a);
  const int n = column_units(a, p, w, threadIdx.x < 64 ? found : nullptr);
  __syncthreads();
  return ColumnUnits{found, n};
}

// Workgroup (column, head) does the units of its column one after the other, and leaves what each of its waves found.  The
// last workgroup writes the plan down where no kernel has before.  (256 threads at least: see chunk_attn_kernel)
template <class C>
__global__ void __launch_bounds__(C::NT > 256 ? C::NT : 256) __attribute__((amdgpu_waves_per_eu(C::WPE))) few_kernel(ChunkAttnArgs a) {
  __shared__ __align__(16) bf16 lds[C::LDS];
  __shared__ ChunkUnit s_units[CO_REQUESTS];
  if (blockIdx.x == (unsigned)a.columns * a.Hkv) {
    if (threadIdx.x < 64) write_plan(a, lane_plan(a));
    return;
  }
  const int h = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv;
  const ColumnUnits us = units_of(a, w, s_units);
  int found = 0;
  for (int i = 0; i < us.n; ++i) {
    const ChunkUnit u = uniform(us.at[i]);
    found |= run_unit<false>(C{}, a, u, h, lds);
  }
  const int bits = (__any(found & UNIT_ODD) ? UNIT_ODD : 0) | (__any(found & UNIT_BAD_PAGE) ? UNIT_BAD_PAGE : 0);
  if ((threadIdx.x & 63) == 0) a.flags[blockIdx.x * C::NW + threadIdx.x / 64] = bits;
}
// The columns some row of which came out infinite or NaN, once more with masked values kept apart (rare).
template <class C>
__global__ void __launch_bounds__(C::NT) few_redo_kernel(ChunkAttnArgs a) {
  __shared__ __align__(16) bf16 lds[C::LDS];
  __shared__ ChunkUnit s_units[CO_REQUESTS];
  const int items = a.columns * a.Hkv, lane = threadIdx.x & 63;
  for (int i0 = blockIdx.x; i0 < items; i0 += gridDim.x * 64) {   // 64 items a round, a lane looks at one
    const long long mine = i0 + (long long)gridDim.x * lane;
    int odd = 0;
    if (mine < items) {
#pragma unroll
      for (int k = 0; k < C::NW; ++k) odd |= a.flags[mine * C::NW + k] & UNIT_ODD;
    }
    for (unsigned long long left = __ballot(odd != 0); left; left &= left - 1) {   // (the same in every wave)
      const int item = i0 + gridDim.x * __builtin_ctzll(left);
      __syncthreads();   // (the last column's units are read)
      const ColumnUnits us = units_of(a, item / a.Hkv, s_units);
      for (int i = 0; i < us.n; ++i) {
        const ChunkUnit u = uniform(us.at[i]);
        run_unit<true>(C{}, a, u, item % a.Hkv, lds);
      }
    }
  }
}

template <class C>
hipError_t launch_few(const ChunkAttnArgs& a, hipStream_t s) {
  const unsigned items = (unsigned)a.columns * a.Hkv;
  hipLaunchKernelGGL(few_kernel<C>, dim3(items + (a.first ? 0 : 1)), dim3(C::NT), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.max_new > 1) {   // (one new token: its rows see the same keys)
    hipLaunchKernelGGL(few_redo_kernel<C>, dim3(std::min(256u, items)), dim3(C::NT), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return launch_merge<typename C::T, C::D>(a, s, C::NW);
}

}  // namespace
}  // namespace hspec
