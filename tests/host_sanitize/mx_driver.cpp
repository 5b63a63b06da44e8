// Runs the entry points of the 4-bit cache and of the logits' adjustment (target_mx_abi.cpp) on the CPU under
// AddressSanitizer and UndefinedBehaviorSanitizer against stand-ins of their launchers, as target_driver.cpp does for those
// of the other caches (whose stand-ins and checks this includes).
#define main target_main
#include "target_driver.cpp"
#undef main

namespace hspec {

hipError_t launch_chunk_append_mx(const ChunkAppendArgs& a, hipStream_t) {
  ++g_launches;
  const size_t pool = (size_t)a.num_pages * a.Hkv * a.ps * (a.D / 2 + a.D / 32);
  touch("qkv", a.qkv, (size_t)a.T * (a.Hq + 2 * a.Hkv) * a.D * (a.in_f32 ? 4 : 2));
  touch("q", a.q, (size_t)a.T * a.Hq * a.D * (a.out_f32 ? 4 : 2));
  touch("k_cache", a.k_cache, pool);
  touch("v_cache", a.v_cache, pool);
  if (a.qw) touch("qw", a.qw, a.D * 4), touch("kw", a.kw, a.D * 4);
  touch("cu", a.cu, (a.B + 1) * 4);
  touch("lens", a.ctx_lens, a.B * 4);
  touch("table", a.page_table, (size_t)a.B * a.max_pages * 4);
  cut("status", a.status, 256);
  return hipSuccess;
}
hipError_t launch_chunk_read_mx(const ChunkAppendArgs& a, void* k, void* v, hipStream_t) {
  ++g_launches;
  const size_t pool = (size_t)a.num_pages * a.Hkv * a.ps * (a.D / 2 + a.D / 32), rows = (size_t)a.T * a.Hkv * a.D * (a.out_f32 ? 4 : 2);
  touch("k", k, rows);
  touch("v", v, rows);
  touch("k_cache", a.k_cache, pool);
  touch("v_cache", a.v_cache, pool);
  touch("cu", a.cu, (a.B + 1) * 4);
  touch("lens", a.ctx_lens, a.B * 4);
  touch("table", a.page_table, (size_t)a.B * a.max_pages * 4);
  cut("status", a.status, 256);
  return hipSuccess;
}
hipError_t launch_chunk_attn_mx(const ChunkAttnArgs& a, hipStream_t) {
  ++g_launches;
  const size_t e = a.f32 ? 4 : 2, pool = (size_t)a.num_pages * a.Hkv * a.ps * (a.D / 2 + a.D / 32);
  touch("q", a.q, (size_t)a.T * a.Hq * a.D * e);
  touch("o", a.o, (size_t)a.T * a.Hq * a.D * e);
  touch("k_cache", a.k_cache, pool);
  touch("v_cache", a.v_cache, pool);
  if (a.k_new) touch("k_new", a.k_new, (size_t)a.T * a.Hkv * a.D * e), touch("v_new", a.v_new, (size_t)a.T * a.Hkv * a.D * e);
  touch("cu", a.cu, (a.B + 1) * 4);
  touch("lens", a.ctx_lens, a.B * 4);
  touch("table", a.page_table, (size_t)a.B * a.max_pages * 4);
  cut("status", a.status, 256);
  cut("queue", a.queue, kChunkClasses * kChunkQueueStride * 4);
  const MxTile t = mx_tile(a);
  if ((a.columns > 0) != (t.rows > 0) || (a.columns > 0) != (a.flags != nullptr)) die("columns");
  if (a.columns) cut("flags", a.flags, (size_t)a.columns * a.Hkv * t.rw * t.kw * 4);
  if (a.first) cut("first", a.first, (size_t)(a.columns + 1) * 4);
  if (!a.columns || a.first) cut("units", a.units, sizeof(ChunkUnit) * a.max_units);
  if (a.columns && !a.first && (a.B > 64 || a.max_units < a.B + a.columns || a.max_slots < a.max_units || a.max_splits < a.B))
    die("a plan of lanes past its workspace");
  cut("splits", a.splits, sizeof(ChunkSplit) * a.max_splits);
  if (a.redo) cut("redo", a.redo, sizeof(int) * a.max_redo);
  if (!a.columns && a.max_new > 1 && !a.redo) die("no redo list");
  const size_t rows = (size_t)a.max_slots * a.Hkv * a.tile_rows;
  cut("part_o", a.part_o, rows * a.D * 4);
  cut("part_ml", a.part_ml, rows * 8);
  return hipSuccess;
}
hipError_t launch_adjust(const AdjustArgs& a, hipStream_t) {
  ++g_launches;
  touch("logits", a.logits, (size_t)a.rows * a.V * (a.in_f32 ? 4 : 2));
  touch("out", a.out, (size_t)a.rows * a.V * (a.out_f32 ? 4 : 2));
  if (a.cu) touch("cu", a.cu, (a.B + 1) * 4);
  if (a.draft_tokens) touch("drafts", a.draft_tokens, (size_t)a.B * a.k * 4);
  if (a.draft_tokens && a.d2t) touch("d2t", a.d2t, (size_t)a.Vd * 4);
  if (a.history) touch("history", a.history, (size_t)a.B * a.max_hist * 4), touch("lens", a.hist_lens, a.B * 4);
  if (a.prompt_lens) touch("prompts", a.prompt_lens, a.B * 4);
  for (const float* p : {a.repetition, a.frequency, a.presence})
    if (p) touch("penalties", p, a.B * 4);
  if (a.n_bias) touch("bias", a.bias, (size_t)a.B * a.n_bias * 4), touch("bias_ids", a.bias_ids, (size_t)a.B * a.n_bias * 4);
  if (a.mask) touch("mask", a.mask, (size_t)a.masks * ((a.V + 31) / 32) * 4);
  if (a.mask_rows) touch("mask_rows", a.mask_rows, (size_t)a.rows * 4);
  if (a.mask && !a.mask_rows && a.masks != a.rows) die("lines of the mask");
  cut("status", a.status, 256);
  return hipSuccess;
}

}  // namespace hspec

namespace {

void mx_chunks(std::mt19937& r) {
  auto pick = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 400; ++i) {
    hspec_chunk_cfg c{};
    c.Hkv = pick(1, 9);
    c.Hq = pick(1, 9) * c.Hkv;
    c.D = pick(0, 1) ? 128 : 64;
    c.B = pick(0, 3) ? pick(1, 20) : pick(60, 90);
    c.T = pick(1, 60);
    c.max_new = pick(1, pick(0, 1) ? 4 : 70);
    c.page_size = 16 << pick(0, 3);
    c.max_pages = pick(1, 40);
    c.num_pages = pick(1, 6);
    c.window = pick(0, 2) ? 0 : pick(1, 300);
    c.dtype = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    c.eps = 1e-6f;
    c.rope_theta = 1e6;
    const size_t e = c.dtype == HSPEC_F32 ? 4 : 2;
    Pool pool;
    const size_t rows = (size_t)c.T * c.Hq * c.D * e, kv = (size_t)c.T * c.Hkv * c.D * e, cache = hspec_mx_cache_bytes(&c);
    if (cache != (size_t)c.num_pages * c.page_size * c.Hkv * (c.D / 2 + c.D / 32)) die("bytes of a cache");
    void *q = pool.get(rows), *o = pool.get(rows), *kc = pool.get(cache), *vc = pool.get(cache), *kn = pool.get(kv), *vn = pool.get(kv);
    auto* cu = (int32_t*)pool.get((c.B + 1) * 4);
    auto* lens = (int32_t*)pool.get(c.B * 4);
    auto* table = (int32_t*)pool.get((size_t)c.B * c.max_pages * 4);
    auto* w = (float*)pool.get(c.D * 4);
    const int max_len = pick(1, 3000);
    size_t n = hspec_chunk_attn_mx_workspace(&c, max_len);
    void* ws = workspace(pool, n);
    const bool dense = pick(0, 1), block = dense && (!c.window || c.max_new <= c.window) && pick(0, 1);
    const void *k1 = dense ? kn : nullptr, *v1 = dense ? vn : nullptr;
    long l0 = g_launches;
    ok("attn", hspec_chunk_attn_mx(&c, q, cu, k1, v1, block, kc, vc, table, lens, max_len, o, ws, n, nullptr), g_launches == l0 + 1);
    refused("attn short workspace", hspec_chunk_attn_mx(&c, q, cu, k1, v1, block, kc, vc, table, lens, max_len, o, ws, n - 1, nullptr),
            HSPEC_ERR_WORKSPACE);
    n = hspec_chunk_append_mx_workspace(&c);
    ws = workspace(pool, n);
    const hspec_dtype in = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    void* qkv = pool.get((size_t)c.T * (c.Hq + 2 * c.Hkv) * c.D * (in == HSPEC_F32 ? 4 : 2));
    const float* gain = pick(0, 1) ? w : nullptr;
    l0 = g_launches;
    ok("append", hspec_chunk_append_mx(&c, in, qkv, gain, gain, cu, lens, q, kc, vc, table, ws, n, nullptr), g_launches == l0 + 1);
    n = hspec_chunk_read_mx_workspace(&c);
    ws = workspace(pool, n);
    l0 = g_launches;
    ok("read", hspec_chunk_read_mx(&c, cu, lens, kc, vc, table, kn, vn, ws, n, nullptr), g_launches == l0 + 1);
    refused("read short workspace", hspec_chunk_read_mx(&c, cu, lens, kc, vc, table, kn, vn, ws, n - 1, nullptr), HSPEC_ERR_WORKSPACE);
  }
}

void adjusts(std::mt19937& r) {
  auto pick = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 400; ++i) {
    hspec_adjust_cfg c{};
    c.B = pick(1, 9);
    c.k = pick(0, 8);
    c.vocab = pick(1, 3000);
    c.draft_vocab = pick(1, c.vocab);
    c.dtype = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    c.out_dtype = pick(0, 1) ? HSPEC_F32 : HSPEC_BF16;
    const bool ragged = pick(0, 1), lines = pick(0, 1), drafts = c.k && pick(0, 1), in_place = c.dtype == c.out_dtype && pick(0, 1);
    c.rows = ragged ? pick(1, c.B * (c.k + 1)) : c.B * (c.k + 1);
    c.max_hist = pick(0, 2) ? pick(1, 300) : 0;
    c.n_bias = pick(0, 2) ? pick(1, 30) : 0;
    c.masks = pick(0, 2) ? (lines ? pick(1, 20) : c.rows) : 0;
    Pool pool;
    auto f = [&](size_t n) { return (float*)pool.get(n * 4, 16); };
    auto t = [&](size_t n) { return (int32_t*)pool.get(n * 4, 16); };
    void* logits = pool.get((size_t)c.rows * c.vocab * (c.dtype == HSPEC_F32 ? 4 : 2), 16);
    void* out = in_place ? logits : pool.get((size_t)c.rows * c.vocab * (c.out_dtype == HSPEC_F32 ? 4 : 2), 16);
    int32_t *cu = ragged ? t(c.B + 1) : nullptr, *tok = drafts ? t((size_t)c.B * c.k) : nullptr;
    int32_t* d2t = pick(0, 1) ? t(c.draft_vocab) : nullptr;
    int32_t *hist = c.max_hist ? t((size_t)c.B * c.max_hist) : nullptr, *lens = hist ? t(c.B) : nullptr, *old = hist && pick(0, 1) ? t(c.B) : nullptr;
    const float *rep = pick(0, 1) ? f(c.B) : nullptr, *fr = pick(0, 1) ? f(c.B) : nullptr, *pr = pick(0, 1) ? f(c.B) : nullptr;
    int32_t* ids = c.n_bias ? t((size_t)c.B * c.n_bias) : nullptr;
    const float* bias = c.n_bias ? f((size_t)c.B * c.n_bias) : nullptr;
    int32_t *mask = c.masks ? t((size_t)c.masks * ((c.vocab + 31) / 32)) : nullptr, *rows = mask && lines ? t(c.rows) : nullptr;
    const size_t n = hspec_adjust_logits_workspace(&c);
    void* ws = workspace(pool, n);
    const long l0 = g_launches;
    ok("adjust", hspec_adjust_logits(&c, logits, cu, tok, d2t, hist, lens, old, rep, fr, pr, ids, bias, mask, rows, out, ws, n, nullptr),
       g_launches == l0 + 1);
    refused("adjust short workspace",
            hspec_adjust_logits(&c, logits, cu, tok, d2t, hist, lens, old, rep, fr, pr, ids, bias, mask, rows, out, ws, n - 1, nullptr),
            HSPEC_ERR_WORKSPACE);
  }
}

}  // namespace

int main() {
  std::mt19937 r(8);
  mx_chunks(r);
  std::printf("append, read and attention\n");
  adjusts(r);
  std::printf("adjustment\n%ld cases passed\n", g_cases);
  return 0;
}
