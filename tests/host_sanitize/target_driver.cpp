// Runs the target-side entry points (target_abi.cpp) on the CPU under AddressSanitizer and
// UndefinedBehaviorSanitizer against stand-ins of their launchers, which check that every extent a kernel would touch
// lies inside the caller's buffers and apart from the other regions of the workspace; checks the attention plan's
// arithmetic (the same functions the plan kernel calls) against the workspace's bounds for random lengths; and that
// rejected calls launch nothing.  Prints one line per group; exits non-zero on the first failed expectation.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "hspec.h"
#include "kernels.h"
#include "target.h"

namespace {

struct Region {
  const char* p;
  size_t n;
};
std::vector<Region> g_bufs;        // what the caller owns
std::vector<Region> g_cut;         // regions of the workspace seen in this call
const char* g_ws = nullptr;
size_t g_ws_n = 0;
long g_launches = 0, g_cases = 0;
char g_msg[512];

[[noreturn]] void die(const char* what) {
  std::fprintf(stderr, "FAIL %s (%s)\n", what, g_msg);
  std::exit(1);
}
void touch(const char* what, const void* p, size_t n) {
  if (n == 0) return;
  const char* c = static_cast<const char*>(p);
  for (const Region& r : g_bufs)
    if (c >= r.p && n <= r.n && (size_t)(c - r.p) <= r.n - n) {
      volatile char sink = c[0];
      sink = c[n - 1];
      (void)sink;
      return;
    }
  die(what);
}
// a region of the workspace: inside it, aligned, apart from the others
void cut(const char* what, const void* p, size_t n) {
  const char* c = static_cast<const char*>(p);
  if (n == 0) return;
  if (!c || c < g_ws || n > g_ws_n || (size_t)(c - g_ws) > g_ws_n - n || (c - g_ws) % 256) die(what);
  for (const Region& r : g_cut)
    if (c < r.p + r.n && r.p < c + n) die(what);
  g_cut.push_back({c, n});
  std::memset(const_cast<char*>(c), 0xa5, n);
}

}  // namespace

namespace hspec {

hspec_status api_fail(hspec_status s, const char* msg) {
  std::snprintf(g_msg, sizeof g_msg, "%s", msg);
  return s;
}
hipError_t launch_chunk_append(const ChunkAppendArgs& a, hipStream_t) {
  ++g_launches;
  const size_t e = a.out_f32 ? 4 : 2;
  touch("qkv", a.qkv, (size_t)a.T * (a.Hq + 2 * a.Hkv) * a.D * (a.in_f32 ? 4 : 2));
  touch("q", a.q, (size_t)a.T * a.Hq * a.D * e);
  touch("k_cache", a.k_cache, (size_t)a.num_pages * a.ps * a.Hkv * a.D * e);
  touch("v_cache", a.v_cache, (size_t)a.num_pages * a.ps * a.Hkv * a.D * e);
  if (a.qw) touch("qw", a.qw, a.D * 4), touch("kw", a.kw, a.D * 4);
  touch("cu", a.cu, (a.B + 1) * 4);
  touch("lens", a.ctx_lens, a.B * 4);
  touch("table", a.page_table, (size_t)a.B * a.max_pages * 4);
  cut("status", a.status, 256);
  return hipSuccess;
}
hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t) {
  ++g_launches;
  const size_t e = a.f32 ? 4 : 2;
  touch("q", a.q, (size_t)a.T * a.Hq * a.D * e);
  touch("o", a.o, (size_t)a.T * a.Hq * a.D * e);
  touch("k_cache", a.k_cache, (size_t)a.num_pages * a.ps * a.Hkv * a.D * e);
  touch("v_cache", a.v_cache, (size_t)a.num_pages * a.ps * a.Hkv * a.D * e);
  touch("cu", a.cu, (a.B + 1) * 4);
  touch("lens", a.ctx_lens, a.B * 4);
  touch("table", a.page_table, (size_t)a.B * a.max_pages * 4);
  cut("status", a.status, 256);
  cut("queue", a.queue, kChunkClasses * kChunkQueueStride * 4);
  cut("units", a.units, sizeof(ChunkUnit) * a.max_units);
  cut("splits", a.splits, sizeof(ChunkSplit) * a.max_splits);
  if (a.redo) cut("redo", a.redo, sizeof(int) * a.max_redo);
  const size_t rows = (size_t)a.max_slots * a.Hkv * a.tile_rows;
  cut("part_o", a.part_o, rows * a.D * 4);
  cut("part_ml", a.part_ml, rows * 8);
  if (a.max_new > 1 && !a.redo) die("no redo list");
  return hipSuccess;
}
hipError_t launch_verify(const VerifyArgs& a, hipStream_t) {
  ++g_launches;
  const size_t rows = (size_t)a.B * (a.k + 1);
  touch("target", a.target, (size_t)a.rows * a.V * (a.f32 ? 4 : 2));
  if (a.draft) touch("draft", a.draft, (size_t)a.B * a.k * a.Vd * 4);
  touch("tokens in", a.draft_tokens, (size_t)a.B * a.k * 4);
  touch("tokens", a.tokens, rows * 4);
  touch("accepted", a.accepted, a.B * 4);
  if (a.cu) touch("cu", a.cu, (a.B + 1) * 4);
  if (a.d2t) touch("d2t", a.d2t, a.Vd * 4);
  if (a.t2d) touch("t2d", a.t2d, a.V * 4);
  if (a.u) touch("u", a.u, (size_t)a.B * a.k * 4), touch("gumbel", a.gumbel, (size_t)a.B * a.V * 4);
  cut("status", a.status, 256);
  cut("stat_t", a.stat_t, (size_t)a.rows * a.pieces_t * 8);
  cut("stat_d", a.stat_d, (size_t)a.B * a.k * a.pieces_d * 8);
  cut("row", a.row, rows * sizeof(VerifyRow));
  cut("count", a.count, rows * kVerifyLine * 4);
  cut("n", a.n, (size_t)a.B * kVerifyLine * 4);
  cut("req", a.req, (size_t)a.B * 8);
  cut("done", a.done, (size_t)a.B * kVerifyLine * 4);
  cut("keys", a.keys, (size_t)a.B * kVerifyLine * 4);
  if (a.pieces_t > 64 || a.pieces_d > 64 || a.pieces_r < 1) die("pieces");
  // a piece fits a workgroup's registers (lengths go in multiples of 256 elements)
  if (((a.V + a.pieces_t - 1) / a.pieces_t + 255) / 256 * 256 * (a.f32 ? 4 : 2) > kVerifyPiece) die("piece of a row");
  if (((a.Vd + a.pieces_d - 1) / a.pieces_d + 255) / 256 * 256 * 4 > kVerifyPiece) die("piece of a draft row");
  return hipSuccess;
}

}  // namespace hspec

extern "C" const char* hipGetErrorString(hipError_t) { return "error"; }

namespace {

struct Pool {
  std::vector<void*> bufs;
  void* get(size_t n, size_t align = 256) {
    void* p = nullptr;
    if (posix_memalign(&p, align, n ? n : 1)) std::abort();
    std::memset(p, 0, n ? n : 1);
    bufs.push_back(p);
    g_bufs.push_back({(char*)p, n});
    return p;
  }
  ~Pool() {
    for (void* p : bufs) std::free(p);
    g_bufs.clear();
  }
};
void* workspace(Pool& pool, size_t n) {
  g_ws = (char*)pool.get(n);
  g_ws_n = n;
  g_cut.clear();
  return (void*)g_ws;
}
void ok(const char* what, hspec_status s, bool launched) {
  static long before = 0;
  if (s != HSPEC_OK || !launched || g_launches != before + 1 || g_msg[0]) die(what);
  before = g_launches;
  ++g_cases;
}
void refused(const char* what, hspec_status s, hspec_status want) {
  static long n = 0;
  const long now = g_launches;
  if (s != want || !g_msg[0]) die(what);
  if (n && now < n) die(what);
  n = now;
  ++g_cases;
}

void chunks(std::mt19937& r) {
  auto pick = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 250; ++i) {
    hspec_chunk_cfg c{};
    const int g = pick(1, 9);
    c.Hkv = pick(1, 9);
    c.Hq = g * c.Hkv;
    c.D = pick(0, 1) ? 128 : 64;
    c.B = pick(1, 20);
    c.T = pick(1, 60);
    c.max_new = pick(1, 70);
    c.page_size = 16 << pick(0, 3);
    c.max_pages = pick(1, 40);
    c.num_pages = pick(1, 6);
    c.window = pick(0, 2) ? 0 : pick(1, 300);
    c.dtype = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    c.eps = 1e-6f;
    c.rope_theta = 1e6;
    const size_t e = c.dtype == HSPEC_F32 ? 4 : 2;
    Pool pool;
    const size_t rows = (size_t)c.T * c.Hq * c.D * e, cache = (size_t)c.num_pages * c.page_size * c.Hkv * c.D * e;
    void *q = pool.get(rows), *o = pool.get(rows), *kc = pool.get(cache), *vc = pool.get(cache);
    auto* cu = (int32_t*)pool.get((c.B + 1) * 4);
    auto* lens = (int32_t*)pool.get(c.B * 4);
    auto* table = (int32_t*)pool.get((size_t)c.B * c.max_pages * 4);
    auto* w = (float*)pool.get(c.D * 4);
    const int max_len = pick(1, 2000);
    size_t n = hspec_chunk_attn_workspace(&c, max_len);
    void* ws = workspace(pool, n);
    long l0 = g_launches;
    ok("attn", hspec_chunk_attn(&c, q, cu, kc, vc, table, lens, max_len, o, ws, n, nullptr), g_launches == l0 + 1);
    refused("attn short workspace", hspec_chunk_attn(&c, q, cu, kc, vc, table, lens, max_len, o, ws, n - 1, nullptr),
            HSPEC_ERR_WORKSPACE);
    n = hspec_chunk_append_workspace(&c);
    ws = workspace(pool, n);
    const hspec_dtype in = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    void* qkv = pool.get((size_t)c.T * (c.Hq + 2 * c.Hkv) * c.D * (in == HSPEC_F32 ? 4 : 2));
    const float* gain = pick(0, 1) ? w : nullptr;
    l0 = g_launches;
    ok("append", hspec_chunk_append(&c, in, qkv, gain, gain, cu, lens, q, kc, vc, table, ws, n, nullptr),
       g_launches == l0 + 1);
    refused("append in place", hspec_chunk_append(&c, in, qkv, gain, gain, cu, lens, qkv, kc, vc, table, ws, n, nullptr),
            HSPEC_ERR_UNSUPPORTED);
  }
}

void verifies(std::mt19937& r) {
  auto pick = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 200; ++i) {
    hspec_verify_cfg c{};
    c.B = pick(1, 9);
    c.k = pick(1, 8);
    c.vocab = pick(1, i % 10 ? 3000 : 20000);
    c.draft_vocab = pick(1, c.vocab);
    c.dtype = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    c.temperature = 0.7f;
    c.draft_temperature = 0.9f;
    const bool ragged = pick(0, 1), sample = pick(0, 1), draft = sample && pick(0, 1), map = pick(0, 1);
    c.rows = ragged ? pick(1, c.B * (c.k + 1)) : c.B * (c.k + 1);
    Pool pool;
    void* target = pool.get((size_t)c.rows * c.vocab * (c.dtype == HSPEC_F32 ? 4 : 2), 16);
    auto f = [&](size_t n) { return (float*)pool.get(n * 4, 16); };
    auto t = [&](size_t n) { return (int32_t*)pool.get(n * 4, 16); };
    const size_t n = hspec_verify_workspace(&c);
    void* ws = workspace(pool, n);
    const long l0 = g_launches;
    const float* dl = draft ? f((size_t)c.B * c.k * c.draft_vocab) : nullptr;
    int32_t *tok = t((size_t)c.B * c.k), *cu = ragged ? t(c.B + 1) : nullptr, *out = t((size_t)c.B * (c.k + 1)), *acc = t(c.B);
    int32_t *d2t = map ? t(c.draft_vocab) : nullptr, *t2d = map && draft ? t(c.vocab) : nullptr;
    const float *u = sample ? f((size_t)c.B * c.k) : nullptr, *gum = sample ? f((size_t)c.B * c.vocab) : nullptr;
    ok("verify", hspec_verify(&c, target, dl, tok, cu, d2t, t2d, u, gum, out, acc, ws, n, nullptr), g_launches == l0 + 1);
    refused("verify short workspace", hspec_verify(&c, target, dl, tok, cu, d2t, t2d, u, gum, out, acc, ws, n - 1, nullptr),
            HSPEC_ERR_WORKSPACE);
  }
  // the largest vocabularies
  for (int f32 = 0; f32 < 2; ++f32) {
    hspec::VerifyArgs a;
    a.B = 1; a.k = 1; a.rows = 2; a.V = a.Vd = 1 << 19; a.f32 = f32;
    hspec::verify_bounds(a);
    if (a.pieces_t > 64 || a.pieces_d > 64) die("pieces of the largest vocabulary");
    ++g_cases;
  }
}

// Units, slots and split tiles of a plan over random lengths stay inside what chunk_bounds reserves.
void plans(std::mt19937& r) {
  auto pick = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 4000; ++i) {
    hspec::ChunkAttnArgs a;
    a.Hkv = 1 << pick(0, 5);
    a.Hq = a.Hkv * pick(1, 16);
    a.D = pick(0, 1) ? 128 : 64;
    a.f32 = pick(0, 3) == 0;
    a.B = pick(1, i % 7 ? 40 : 400);
    const int top = 1 << pick(0, 10), g = a.Hq / a.Hkv;
    const int longest = 1 << pick(0, 17);
    std::vector<int> n(a.B), L(a.B);
    a.max_new = 1;
    for (int b = 0; b < a.B; ++b) {
      n[b] = pick(0, top);
      L[b] = pick(0, 4) ? pick(0, longest) : longest;
      a.T += n[b];
      a.max_new = std::max(a.max_new, n[b]);
      a.cap = std::max(a.cap, L[b] + n[b]);
    }
    a.T = std::max(a.T, 1);
    a.window = pick(0, 2) ? 0 : pick(1, longest);
    hspec::chunk_bounds(a);
    unsigned long long keys = 0;
    std::vector<int> lens;
    for (int b = 0; b < a.B; ++b)
      for (int c0 = 0; c0 < n[b] * g; c0 += a.tile_rows) {
        const int t0 = c0 / g, t1 = (std::min(c0 + a.tile_rows, n[b] * g) - 1) / g;
        const int k0 = a.window ? std::max(L[b] + t0 - a.window + 1, 0) / a.key_tile * a.key_tile : 0;
        lens.push_back(std::max(L[b] + t1 + 1 - k0, 0));
        keys += lens.back();
      }
    const int S = hspec::chunk_unit_keys(a, keys, (int)lens.size());
    long long units = 0, slots = 0, splits = 0;
    for (int len : lens) {
      int q;
      const int p = hspec::chunk_pieces(len, S, a.key_tile, q);
      if (p < 1 || (long long)p * q < len || (p > 1 && ((long long)(p - 1) * q >= len || q % a.key_tile))) die("pieces of a tile");
      units += p;
      if (p > 1) slots += p, ++splits;
    }
    if (units > a.max_units || slots > a.max_slots || splits > a.max_splits) die("plan past its workspace");
    ++g_cases;
  }
}

}  // namespace

int main() {
  std::mt19937 r(7);
  chunks(r);
  std::printf("append and attention\n");
  verifies(r);
  std::printf("verification\n");
  plans(r);
  std::printf("plans\n%ld cases passed\n", g_cases);
  return 0;
}
