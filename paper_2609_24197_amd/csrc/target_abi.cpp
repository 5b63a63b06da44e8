// C ABI of the target's side of a step (append, chunk attention, verification): argument checks, workspace
// layout and launches.  Host code only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "hspec.h"
#include "kernels.h"
#include "target.h"

#define HSPEC_API extern "C" __attribute__((visibility("default")))

namespace {

constexpr size_t ALIGN = 256;

template <class... A>
hspec_status fail(hspec_status s, const char* fmt, A... a) {
  char msg[256];
  snprintf(msg, sizeof msg, fmt, a...);
  return hspec::api_fail(s, msg);
}
void clear_err() { hspec::api_fail(HSPEC_OK, ""); }
hspec_status launched(hipError_t e) {
  return e == hipSuccess ? HSPEC_OK : hspec::api_fail(HSPEC_ERR_LAUNCH, hipGetErrorString(e));
}

// Bump allocator over the caller's workspace.  With base == nullptr it only measures.
struct Arena {
  char* base = nullptr;
  size_t off = 0;
  template <class T>
  T* take(size_t count) {
    const size_t o = (off + ALIGN - 1) / ALIGN * ALIGN;
    off = o + count * sizeof(T);
    return base ? reinterpret_cast<T*>(base + o) : nullptr;
  }
  size_t size() const { return (off + ALIGN - 1) / ALIGN * ALIGN; }
};

hspec_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws) return fail(HSPEC_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % ALIGN) return fail(HSPEC_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (have < need) return fail(HSPEC_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", have, need);
  return HSPEC_OK;
}

// Rows are read and written 16 bytes at a time.
hspec_status check_aligned(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(HSPEC_ERR_UNSUPPORTED, "a tensor is not 16-byte aligned");
  return HSPEC_OK;
}

// Memory of an argument; an extent past what can be addressed counts as 2^62 bytes.
struct Span {
  const void* p;
  size_t n;
};
Span span(const void* p, std::initializer_list<size_t> dims) {
  unsigned __int128 n = 1;
  for (size_t d : dims) n = std::min(n * d, (unsigned __int128)1 << 62);
  return Span{p, (size_t)n};
}
// What a call writes must lie over nothing else that it is given.
hspec_status check_apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  auto over = [](const Span& x, const Span& y) {
    const uintptr_t a = (uintptr_t)x.p, b = (uintptr_t)y.p;
    return a && b && (a < b ? b - a < x.n : a - b < y.n);
  };
  for (const Span* x = outs.begin(); x != outs.end(); ++x) {
    bool bad = false;
    for (const Span& y : ins) bad |= over(*x, y);
    for (const Span* y = x + 1; y != outs.end(); ++y) bad |= over(*x, *y);
    if (bad) return fail(HSPEC_ERR_UNSUPPORTED, "an output or the workspace lies over another argument");
  }
  return HSPEC_OK;
}
size_t size_of(hspec_dtype d) { return d == HSPEC_F32 ? 4 : 2; }

bool dtype_ok(hspec_dtype d) { return d == HSPEC_BF16 || d == HSPEC_F32; }

hspec_status check_chunk(const hspec_chunk_cfg* c) {
  if (!c) return fail(HSPEC_ERR_NULL, "chunk config is NULL");
  if (!dtype_ok(c->dtype)) return fail(HSPEC_ERR_DTYPE, "unknown dtype %d", (int)c->dtype);
  if (c->B <= 0 || c->T <= 0 || c->max_new <= 0 || c->Hq <= 0 || c->Hkv <= 0 || c->D <= 0 || c->page_size <= 0 ||
      c->max_pages <= 0 || c->num_pages <= 0)
    return fail(HSPEC_ERR_SHAPE, "non-positive chunk dimension");
  if (c->Hq % c->Hkv) return fail(HSPEC_ERR_SHAPE, "Hq %% Hkv != 0 (Hq=%d, Hkv=%d)", c->Hq, c->Hkv);
  if (c->window < 0) return fail(HSPEC_ERR_SHAPE, "window < 0");
  if (c->D != 64 && c->D != 128) return fail(HSPEC_ERR_UNSUPPORTED, "D must be 64 or 128, got %d", c->D);
  if (c->page_size < 16 || (c->page_size & (c->page_size - 1)))
    return fail(HSPEC_ERR_UNSUPPORTED, "page_size must be a power of two >= 16, got %d", c->page_size);
  if (c->B > 32767) return fail(HSPEC_ERR_UNSUPPORTED, "B must be <= 32767");
  if (c->Hq > 4096) return fail(HSPEC_ERR_UNSUPPORTED, "Hq must be <= 4096");
  if ((long long)c->T * c->Hq > (1LL << 28))   // (units, rows and work items stay inside 31 bits)
    return fail(HSPEC_ERR_UNSUPPORTED, "T * Hq must be <= 2^28");
  return HSPEC_OK;
}

Span cache_span(const hspec_chunk_cfg& c, const void* p) {
  return span(p, {(size_t)c.num_pages, (size_t)c.page_size, (size_t)c.Hkv, (size_t)c.D, size_of(c.dtype)});
}
Span rows_span(const hspec_chunk_cfg& c, const void* p) {
  return span(p, {(size_t)c.T, (size_t)c.Hq, (size_t)c.D, size_of(c.dtype)});
}
Span ints_span(const void* p, size_t n, size_t m = 1) { return span(p, {n, m, 4}); }

int positions(const hspec_chunk_cfg& c) {
  return (int)std::min((long long)c.max_pages * c.page_size, (long long)hspec::kMaxPositions);
}

}  // namespace

// ------------------------------------------------------------------------------ append

HSPEC_API size_t hspec_chunk_append_workspace(const hspec_chunk_cfg* cfg) { return cfg ? ALIGN : 0; }

HSPEC_API hspec_status hspec_chunk_append(const hspec_chunk_cfg* cfg, hspec_dtype qkv_dtype, const void* qkv,
                                          const float* q_norm_w, const float* k_norm_w, const int32_t* cu_new,
                                          const int32_t* ctx_lens, void* q, void* k_cache, void* v_cache,
                                          const int32_t* page_table, void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_chunk(cfg)) return s;
  if (!dtype_ok(qkv_dtype)) return fail(HSPEC_ERR_DTYPE, "unknown qkv dtype %d", (int)qkv_dtype);
  if (!qkv || !cu_new || !ctx_lens || !q || !k_cache || !v_cache || !page_table)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (!q_norm_w != !k_norm_w) return fail(HSPEC_ERR_NULL, "only one of q_norm_w and k_norm_w is NULL");
  if (!(cfg->rope_theta > 0.)) return fail(HSPEC_ERR_SHAPE, "rope_theta must be positive");
  if (hspec_status s = check_aligned({qkv, q, k_cache, v_cache})) return s;
  const size_t need = hspec_chunk_append_workspace(cfg);
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  const hspec_chunk_cfg& c = *cfg;
  if (hspec_status s = check_apart({rows_span(c, q), cache_span(c, k_cache), cache_span(c, v_cache), Span{workspace, need}},
                                   {span(qkv, {(size_t)c.T, (size_t)(c.Hq + 2 * c.Hkv), (size_t)c.D, size_of(qkv_dtype)}),
                                    ints_span(q_norm_w, c.D), ints_span(k_norm_w, c.D), ints_span(cu_new, c.B + 1),
                                    ints_span(ctx_lens, c.B), ints_span(page_table, c.B, c.max_pages)}))
    return s;
  hspec::ChunkAppendArgs a;
  a.qkv = qkv; a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.qw = q_norm_w; a.kw = k_norm_w;
  a.cu = cu_new; a.ctx_lens = ctx_lens; a.page_table = page_table;
  a.B = c.B; a.T = c.T; a.max_new = c.max_new; a.Hq = c.Hq; a.Hkv = c.Hkv; a.D = c.D; a.ps = c.page_size;
  a.max_pages = c.max_pages; a.num_pages = c.num_pages; a.cap = positions(c);
  a.eps = c.eps; a.rope_theta = c.rope_theta;
  a.status = static_cast<int*>(workspace);
  a.in_f32 = qkv_dtype == HSPEC_F32; a.out_f32 = c.dtype == HSPEC_F32;
  return launched(hspec::launch_chunk_append(a, (hipStream_t)stream));
}

// --------------------------------------------------------------------------- attention

static void plan_chunk_attn(Arena& ar, const hspec_chunk_cfg& c, int max_len, hspec::ChunkAttnArgs& a) {
  a.B = c.B; a.T = c.T; a.max_new = std::min(c.max_new, c.T); a.Hq = c.Hq; a.Hkv = c.Hkv; a.D = c.D;
  a.ps = c.page_size; a.max_pages = c.max_pages; a.num_pages = c.num_pages;
  a.window = c.window; a.cap = std::min(max_len, positions(c)); a.f32 = c.dtype == HSPEC_F32;
  hspec::chunk_bounds(a);
  a.status = ar.take<int>(64);
  a.queue = ar.take<int>(hspec::kChunkClasses * hspec::kChunkQueueStride);
  a.units = ar.take<hspec::ChunkUnit>(a.max_units);
  a.splits = ar.take<hspec::ChunkSplit>(a.max_splits);
  // one new token a request: its rows see the same keys, and the others' places in its tiles are zeros
  if (a.max_new > 1) a.redo = ar.take<int>(a.max_redo);
  const size_t rows = (size_t)a.max_slots * c.Hkv * a.tile_rows;
  a.part_o = ar.take<float>(rows * c.D);
  a.part_ml = ar.take<float>(rows * 2);
}

HSPEC_API size_t hspec_chunk_attn_workspace(const hspec_chunk_cfg* cfg, int max_len) {
  if (!cfg || max_len <= 0 || check_chunk(cfg)) return 0;
  Arena ar;
  hspec::ChunkAttnArgs a;
  plan_chunk_attn(ar, *cfg, max_len, a);
  return ar.size();
}

HSPEC_API hspec_status hspec_chunk_attn(const hspec_chunk_cfg* cfg, const void* q, const int32_t* cu_new,
                                        const void* k_cache, const void* v_cache, const int32_t* page_table,
                                        const int32_t* ctx_lens, int max_len, void* o, void* workspace, size_t ws_bytes,
                                        void* stream) {
  clear_err();
  if (hspec_status s = check_chunk(cfg)) return s;
  if (max_len <= 0) return fail(HSPEC_ERR_SHAPE, "max_len must be positive");
  if (!(cfg->scale >= 0.f && cfg->scale <= 1e30f)) return fail(HSPEC_ERR_SHAPE, "scale must be finite and not negative");
  if (!q || !cu_new || !k_cache || !v_cache || !page_table || !ctx_lens || !o)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (hspec_status s = check_aligned({q, k_cache, v_cache, o})) return s;
  const size_t need = hspec_chunk_attn_workspace(cfg, max_len);
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  if (hspec_status s = check_apart({rows_span(*cfg, o), Span{workspace, need}},
                                   {rows_span(*cfg, q), cache_span(*cfg, k_cache), cache_span(*cfg, v_cache),
                                    ints_span(cu_new, cfg->B + 1), ints_span(ctx_lens, cfg->B),
                                    ints_span(page_table, cfg->B, cfg->max_pages)}))
    return s;
  Arena ar{(char*)workspace};
  hspec::ChunkAttnArgs a;
  plan_chunk_attn(ar, *cfg, max_len, a);
  a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.o = o;
  a.cu = cu_new; a.ctx_lens = ctx_lens; a.page_table = page_table;
  const double scale = cfg->scale > 0.f ? cfg->scale : 1. / std::sqrt((double)cfg->D);
  a.scale_log2 = (float)(scale * 1.4426950408889634074);
  return launched(hspec::launch_chunk_attn(a, (hipStream_t)stream));
}

// ------------------------------------------------------------------------ verification

static hspec_status check_verify(const hspec_verify_cfg* c) {
  if (!c) return fail(HSPEC_ERR_NULL, "verification config is NULL");
  if (!dtype_ok(c->dtype)) return fail(HSPEC_ERR_DTYPE, "unknown dtype %d", (int)c->dtype);
  if (c->B <= 0 || c->k <= 0 || c->rows <= 0 || c->vocab <= 0 || c->draft_vocab <= 0)
    return fail(HSPEC_ERR_SHAPE, "non-positive verification dimension");
  if (c->draft_vocab > c->vocab)
    return fail(HSPEC_ERR_SHAPE, "the draft vocabulary (%d) is larger than the target's (%d)", c->draft_vocab, c->vocab);
  if (c->vocab > (1 << 19) || c->B > 32767 || c->k > 4096 || (long long)c->B * (c->k + 1) > (1 << 22) || c->rows > (1 << 22))
    return fail(HSPEC_ERR_UNSUPPORTED, "verification too large");
  return HSPEC_OK;
}

// log2(e) / T is positive and finite.
static bool temperature_ok(float t) { return t > 0.f && std::isfinite(t) && std::isfinite((float)(1.5 / t)); }

static void plan_verify(Arena& ar, const hspec_verify_cfg& c, hspec::VerifyArgs& a) {
  a.B = c.B; a.k = c.k; a.rows = c.rows; a.V = c.vocab; a.Vd = c.draft_vocab; a.f32 = c.dtype == HSPEC_F32;
  hspec::verify_bounds(a);
  a.status = ar.take<int>(64);
  const size_t rows = (size_t)c.B * (c.k + 1);
  a.keys = ar.take<unsigned long long>((size_t)c.B * hspec::verify_key_stride(a.pieces_r));
  a.stat_t = ar.take<unsigned long long>((size_t)c.rows * a.pieces_t);
  a.stat_d = ar.take<unsigned long long>((size_t)c.B * c.k * a.pieces_d);
  a.row = ar.take<hspec::VerifyRow>(rows);
  a.count = ar.take<int>(rows * hspec::kVerifyLine);
  a.n = ar.take<int>((size_t)c.B * hspec::kVerifyLine);
  a.req = ar.take<int2>(c.B);
  a.done = ar.take<int>((size_t)c.B * hspec::kVerifyLine);
}

HSPEC_API size_t hspec_verify_workspace(const hspec_verify_cfg* cfg) {
  if (!cfg || check_verify(cfg)) return 0;
  Arena ar;
  hspec::VerifyArgs a;
  plan_verify(ar, *cfg, a);
  return ar.size();
}

HSPEC_API hspec_status hspec_verify(const hspec_verify_cfg* cfg, const void* target_logits, const float* draft_logits,
                                    const int32_t* draft_tokens, const int32_t* cu_rows, const int32_t* d2t,
                                    const int32_t* t2d, const float* u, const float* gumbel, int32_t* tokens,
                                    int32_t* n_accepted, void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_verify(cfg)) return s;
  if (!target_logits || !draft_tokens || !tokens || !n_accepted)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (!u != !gumbel) return fail(HSPEC_ERR_NULL, "sampling needs both u and gumbel, greedy verification neither");
  if (!u && draft_logits) return fail(HSPEC_ERR_UNSUPPORTED, "greedy verification takes no draft logits");
  if (draft_logits && !d2t != !t2d) return fail(HSPEC_ERR_NULL, "draft logits need both vocabulary maps or neither");
  if (u && !temperature_ok(cfg->temperature))
    return fail(HSPEC_ERR_SHAPE, "sampling needs a finite temperature > 0");
  if (draft_logits && !temperature_ok(cfg->draft_temperature))
    return fail(HSPEC_ERR_SHAPE, "draft logits need a finite draft_temperature > 0");
  if (!cu_rows && cfg->rows != (long long)cfg->B * (cfg->k + 1))
    return fail(HSPEC_ERR_SHAPE, "without cu_rows, rows must be B * (k + 1)");
  const size_t need = hspec_verify_workspace(cfg), B = cfg->B, k = cfg->k, V = cfg->vocab, Vd = cfg->draft_vocab;
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  if (hspec_status s = check_apart({ints_span(tokens, B, k + 1), ints_span(n_accepted, B), Span{workspace, need}},
                                   {span(target_logits, {(size_t)cfg->rows, V, size_of(cfg->dtype)}),
                                    span(draft_logits, {B, k, Vd, 4}), ints_span(draft_tokens, B, k), ints_span(cu_rows, B + 1),
                                    ints_span(d2t, Vd), ints_span(t2d, V), ints_span(u, B, k), ints_span(gumbel, B, V)}))
    return s;
  Arena ar{(char*)workspace};
  hspec::VerifyArgs a;
  plan_verify(ar, *cfg, a);
  a.u = u;
  a.target = target_logits; a.draft = draft_logits; a.draft_tokens = draft_tokens; a.cu = cu_rows; a.d2t = d2t;
  a.t2d = t2d; a.gumbel = gumbel; a.tokens = tokens; a.accepted = n_accepted;
  const double log2e = 1.4426950408889634074;
  a.c64_t = u ? log2e / cfg->temperature : 1.;
  a.c64_d = draft_logits ? log2e / cfg->draft_temperature : 1.;
  a.c_t = (float)a.c64_t;
  a.c_d = (float)a.c64_d;
  return launched(hspec::launch_verify(a, (hipStream_t)stream));
}
