// C ABI of the 4-bit cache (append, read, attention) and of the logits' adjustment: argument checks, workspace layout
// and launches.  Host code only.
#include "mx_layout.h"
#include "target_check.h"

namespace {

// Kernels address a head's part of a page with 31 bits, and what they leave out with an offset past its end (BUF_OOB).
hspec_status check_mx(const hspec_chunk_cfg* c) {
  if (hspec_status s = check_chunk(c)) return s;
  if (hspec::mx_head_bytes(c->page_size, c->D) >= 1ull << 31)
    return fail(HSPEC_ERR_UNSUPPORTED, "a head's part of a page must be below 2^31 bytes (page_size=%d)", c->page_size);
  return HSPEC_OK;
}

Span mx_span(const hspec_chunk_cfg& c, const void* p) {
  return span(p, {(size_t)c.num_pages, (size_t)c.page_size, (size_t)c.Hkv, (size_t)c.D / 32 * 17});
}
Span kv_span(const hspec_chunk_cfg& c, const void* p) {
  return span(p, {(size_t)c.T, (size_t)c.Hkv, (size_t)c.D, size_of(c.dtype)});
}

hspec::ChunkAppendArgs batch_args(const hspec_chunk_cfg& c, const int32_t* cu, const int32_t* lens, const void* k_cache,
                                  const void* v_cache, const int32_t* table, void* workspace) {
  hspec::ChunkAppendArgs a;
  a.k_cache = const_cast<void*>(k_cache); a.v_cache = const_cast<void*>(v_cache);
  a.cu = cu; a.ctx_lens = lens; a.page_table = table;
  a.B = c.B; a.T = c.T; a.max_new = c.max_new; a.Hq = c.Hq; a.Hkv = c.Hkv; a.D = c.D; a.ps = c.page_size;
  a.max_pages = c.max_pages; a.num_pages = c.num_pages; a.cap = positions(c);
  a.eps = c.eps; a.rope_theta = c.rope_theta;
  a.status = static_cast<int*>(workspace);
  a.out_f32 = c.dtype == HSPEC_F32;
  return a;
}

}  // namespace

HSPEC_API size_t hspec_mx_cache_bytes(const hspec_chunk_cfg* cfg) {
  return !cfg || check_mx(cfg) ? 0 : mx_span(*cfg, nullptr).n;
}

// ------------------------------------------------------------------------------ append

HSPEC_API size_t hspec_chunk_append_mx_workspace(const hspec_chunk_cfg* cfg) { return cfg ? ALIGN : 0; }

HSPEC_API hspec_status hspec_chunk_append_mx(const hspec_chunk_cfg* cfg, hspec_dtype qkv_dtype, const void* qkv,
                                             const float* q_norm_w, const float* k_norm_w, const int32_t* cu_new,
                                             const int32_t* ctx_lens, void* q, void* k_cache, void* v_cache,
                                             const int32_t* page_table, void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_mx(cfg)) return s;
  if (!dtype_ok(qkv_dtype)) return fail(HSPEC_ERR_DTYPE, "unknown qkv dtype %d", (int)qkv_dtype);
  if (!qkv || !cu_new || !ctx_lens || !q || !k_cache || !v_cache || !page_table)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (!q_norm_w != !k_norm_w) return fail(HSPEC_ERR_NULL, "only one of q_norm_w and k_norm_w is NULL");
  if (!(cfg->rope_theta > 0.)) return fail(HSPEC_ERR_SHAPE, "rope_theta must be positive");
  if (hspec_status s = check_aligned({qkv, q, k_cache, v_cache})) return s;
  const size_t need = hspec_chunk_append_mx_workspace(cfg);
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  const hspec_chunk_cfg& c = *cfg;
  if (hspec_status s = check_apart({rows_span(c, q), mx_span(c, k_cache), mx_span(c, v_cache), Span{workspace, need}},
                                   {span(qkv, {(size_t)c.T, (size_t)(c.Hq + 2 * c.Hkv), (size_t)c.D, size_of(qkv_dtype)}),
                                    ints_span(q_norm_w, c.D), ints_span(k_norm_w, c.D), ints_span(cu_new, c.B + 1),
                                    ints_span(ctx_lens, c.B), ints_span(page_table, c.B, c.max_pages)}))
    return s;
  hspec::ChunkAppendArgs a = batch_args(c, cu_new, ctx_lens, k_cache, v_cache, page_table, workspace);
  a.qkv = qkv; a.q = q; a.qw = q_norm_w; a.kw = k_norm_w;
  a.in_f32 = qkv_dtype == HSPEC_F32;
  return launched(hspec::launch_chunk_append_mx(a, (hipStream_t)stream));
}

// -------------------------------------------------------------------------------- read

HSPEC_API size_t hspec_chunk_read_mx_workspace(const hspec_chunk_cfg* cfg) { return cfg ? ALIGN : 0; }

HSPEC_API hspec_status hspec_chunk_read_mx(const hspec_chunk_cfg* cfg, const int32_t* cu_new, const int32_t* ctx_lens,
                                           const void* k_cache, const void* v_cache, const int32_t* page_table, void* k,
                                           void* v, void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_mx(cfg)) return s;
  if (!cu_new || !ctx_lens || !k_cache || !v_cache || !page_table || !k || !v)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (hspec_status s = check_aligned({k_cache, v_cache, k, v})) return s;
  const size_t need = hspec_chunk_read_mx_workspace(cfg);
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  const hspec_chunk_cfg& c = *cfg;
  if (hspec_status s = check_apart({kv_span(c, k), kv_span(c, v), Span{workspace, need}},
                                   {mx_span(c, k_cache), mx_span(c, v_cache), ints_span(cu_new, c.B + 1),
                                    ints_span(ctx_lens, c.B), ints_span(page_table, c.B, c.max_pages)}))
    return s;
  const hspec::ChunkAppendArgs a = batch_args(c, cu_new, ctx_lens, k_cache, v_cache, page_table, workspace);
  return launched(hspec::launch_chunk_read_mx(a, k, v, (hipStream_t)stream));
}

// --------------------------------------------------------------------------- attention

static void plan_chunk_attn_mx(Arena& ar, const hspec_chunk_cfg& c, int max_len, hspec::ChunkAttnArgs& a) {
  a.B = c.B; a.T = c.T; a.max_new = std::min(c.max_new, c.T); a.Hq = c.Hq; a.Hkv = c.Hkv; a.D = c.D;
  a.ps = c.page_size; a.max_pages = c.max_pages; a.num_pages = c.num_pages;
  a.window = c.window; a.f32 = c.dtype == HSPEC_F32;
  // (positions beside the cache have no page, so the table does not bound them; one workspace serves both ways)
  a.cap = std::min(max_len, hspec::kMaxPositions);
  hspec::mx_bounds(a);
  a.status = ar.take<int>(64);
  a.queue = ar.take<int>(hspec::kChunkClasses * hspec::kChunkQueueStride);
  if (a.columns) a.flags = ar.take<int>(a.max_flags);
  if (!a.columns || a.B > 64) {
    if (a.columns) a.first = ar.take<int>((size_t)a.columns + 1);
    a.units = ar.take<hspec::ChunkUnit>(a.max_units);
  }
  a.splits = ar.take<hspec::ChunkSplit>(a.max_splits);
  if (!a.columns && a.max_new > 1) a.redo = ar.take<int>(a.max_redo);   // (one new token: its rows see the same keys)
  const size_t rows = (size_t)a.max_slots * c.Hkv * a.tile_rows;
  a.part_o = ar.take<float>(rows * c.D);
  a.part_ml = ar.take<float>(rows * 2);
}

HSPEC_API size_t hspec_chunk_attn_mx_workspace(const hspec_chunk_cfg* cfg, int max_len) {
  if (!cfg || max_len <= 0 || check_mx(cfg)) return 0;
  Arena ar;
  hspec::ChunkAttnArgs a;
  plan_chunk_attn_mx(ar, *cfg, max_len, a);
  return ar.size();
}

HSPEC_API hspec_status hspec_chunk_attn_mx(const hspec_chunk_cfg* cfg, const void* q, const int32_t* cu_new,
                                           const void* k_new, const void* v_new, unsigned flags, const void* k_cache,
                                           const void* v_cache, const int32_t* page_table, const int32_t* ctx_lens,
                                           int max_len, void* o, void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_mx(cfg)) return s;
  if (max_len <= 0) return fail(HSPEC_ERR_SHAPE, "max_len must be positive");
  if (!(cfg->scale >= 0.f && cfg->scale <= 1e30f)) return fail(HSPEC_ERR_SHAPE, "scale must be finite and not negative");
  if (!q || !cu_new || !k_cache || !v_cache || !page_table || !ctx_lens || !o)
    return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (!k_new != !v_new) return fail(HSPEC_ERR_NULL, "only one of k_new and v_new is NULL");
  if (flags & ~(unsigned)HSPEC_CHUNK_BLOCK) return fail(HSPEC_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
  const bool block = flags & HSPEC_CHUNK_BLOCK;
  if (block && !k_new) return fail(HSPEC_ERR_NULL, "HSPEC_CHUNK_BLOCK needs k_new and v_new");
  if (block && cfg->window > 0 && cfg->max_new > cfg->window)
    return fail(HSPEC_ERR_UNSUPPORTED, "HSPEC_CHUNK_BLOCK needs max_new <= window");
  if (hspec_status s = check_aligned({q, k_new, v_new, k_cache, v_cache, o})) return s;
  const size_t need = hspec_chunk_attn_mx_workspace(cfg, max_len);
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  const hspec_chunk_cfg& c = *cfg;
  if (hspec_status s = check_apart({rows_span(c, o), Span{workspace, need}},
                                   {rows_span(c, q), kv_span(c, k_new), kv_span(c, v_new), mx_span(c, k_cache),
                                    mx_span(c, v_cache), ints_span(cu_new, c.B + 1), ints_span(ctx_lens, c.B),
                                    ints_span(page_table, c.B, c.max_pages)}))
    return s;
  Arena ar{(char*)workspace};
  hspec::ChunkAttnArgs a;
  plan_chunk_attn_mx(ar, c, max_len, a);
  a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.o = o; a.k_new = k_new; a.v_new = v_new;
  a.cu = cu_new; a.ctx_lens = ctx_lens; a.page_table = page_table;
  a.block = block;
  a.held = positions(c);
  if (!k_new) a.cap = std::min(a.cap, a.held);
  const double scale = c.scale > 0.f ? c.scale : 1. / std::sqrt((double)c.D);
  a.scale_log2 = (float)(scale * 1.4426950408889634074);
  return launched(hspec::launch_chunk_attn_mx(a, (hipStream_t)stream));
}

// -------------------------------------------------------------------------- adjustment

static hspec_status check_adjust(const hspec_adjust_cfg* c) {
  if (!c) return fail(HSPEC_ERR_NULL, "adjustment config is NULL");
  if (!dtype_ok(c->dtype) || !dtype_ok(c->out_dtype))
    return fail(HSPEC_ERR_DTYPE, "unknown dtype %d or %d", (int)c->dtype, (int)c->out_dtype);
  if (c->B <= 0 || c->k < 0 || c->rows <= 0 || c->vocab <= 0 || c->draft_vocab < 0 || c->max_hist < 0 || c->n_bias < 0 ||
      c->masks < 0)
    return fail(HSPEC_ERR_SHAPE, "a dimension of the adjustment is negative, or B, rows or vocab is 0");
  if (c->vocab > (1 << 19) || c->draft_vocab > (1 << 19) || c->B > 32767 || c->k > 4096 ||
      (long long)c->B * (c->k + 1) > (1 << 22) || c->rows > (1 << 22) || c->max_hist > (1 << 24) || c->n_bias > (1 << 20) ||
      c->masks > (1 << 22))
    return fail(HSPEC_ERR_UNSUPPORTED, "adjustment too large");
  return HSPEC_OK;
}

HSPEC_API size_t hspec_adjust_logits_workspace(const hspec_adjust_cfg* cfg) { return !cfg || check_adjust(cfg) ? 0 : ALIGN; }

HSPEC_API hspec_status hspec_adjust_logits(const hspec_adjust_cfg* cfg, const void* logits, const int32_t* cu_rows,
                                           const int32_t* draft_tokens, const int32_t* d2t, const int32_t* history,
                                           const int32_t* hist_lens, const int32_t* prompt_lens, const float* repetition,
                                           const float* frequency, const float* presence, const int32_t* bias_ids,
                                           const float* bias, const int32_t* mask, const int32_t* mask_rows, void* out,
                                           void* workspace, size_t ws_bytes, void* stream) {
  clear_err();
  if (hspec_status s = check_adjust(cfg)) return s;
  const hspec_adjust_cfg& c = *cfg;
  if (!logits || !out) return fail(HSPEC_ERR_NULL, "an input or output pointer is NULL");
  if (draft_tokens && (c.k == 0 || c.draft_vocab == 0)) return fail(HSPEC_ERR_SHAPE, "draft tokens need k and draft_vocab > 0");
  if (!history != (c.max_hist == 0) || !history != !hist_lens)
    return fail(HSPEC_ERR_NULL, "history, hist_lens and max_hist come together");
  if (prompt_lens && !history) return fail(HSPEC_ERR_NULL, "prompt_lens is given without a history");
  if (!bias_ids != !bias || !bias != (c.n_bias == 0)) return fail(HSPEC_ERR_NULL, "bias_ids, bias and n_bias come together");
  if (!mask != (c.masks == 0)) return fail(HSPEC_ERR_NULL, "mask and masks come together");
  if (mask_rows && !mask) return fail(HSPEC_ERR_NULL, "mask_rows is given without a mask");
  if (mask && !mask_rows && c.masks != c.rows) return fail(HSPEC_ERR_SHAPE, "without mask_rows, masks must be rows");
  if (!cu_rows && c.rows != (long long)c.B * (c.k + 1))
    return fail(HSPEC_ERR_SHAPE, "without cu_rows, rows must be B * (k + 1)");
  if ((uintptr_t)logits % size_of(c.dtype) || (uintptr_t)out % size_of(c.out_dtype))
    return fail(HSPEC_ERR_UNSUPPORTED, "logits or out is not aligned to its type");
  if (out == logits && c.dtype != c.out_dtype) return fail(HSPEC_ERR_UNSUPPORTED, "in place, out_dtype must be dtype");
  const size_t need = hspec_adjust_logits_workspace(cfg), B = c.B, V = c.vocab, rows = c.rows;
  if (hspec_status s = check_ws(workspace, ws_bytes, need)) return s;
  if (hspec_status s = check_apart({span(out, {rows, V, size_of(c.out_dtype)}), Span{workspace, need}},
                                   {span(out == logits ? nullptr : logits, {rows, V, size_of(c.dtype)}),
                                    ints_span(cu_rows, B + 1), ints_span(draft_tokens, B, c.k), ints_span(d2t, c.draft_vocab),
                                    ints_span(history, B, c.max_hist), ints_span(hist_lens, B), ints_span(prompt_lens, B),
                                    ints_span(repetition, B), ints_span(frequency, B), ints_span(presence, B),
                                    ints_span(bias_ids, B, c.n_bias), ints_span(bias, B, c.n_bias),
                                    ints_span(mask, c.masks, (V + 31) / 32), ints_span(mask_rows, rows)}))
    return s;
  hspec::AdjustArgs a;
  a.logits = logits; a.out = out; a.cu = cu_rows; a.draft_tokens = draft_tokens; a.d2t = d2t;
  a.history = history; a.hist_lens = hist_lens; a.prompt_lens = prompt_lens;
  a.repetition = repetition; a.frequency = frequency; a.presence = presence;
  a.bias_ids = bias_ids; a.bias = bias; a.mask = reinterpret_cast<const uint32_t*>(mask); a.mask_rows = mask_rows;
  a.B = c.B; a.k = c.k; a.rows = c.rows; a.V = c.vocab; a.Vd = c.draft_vocab; a.max_hist = c.max_hist; a.n_bias = c.n_bias;
  a.masks = c.masks; a.in_f32 = c.dtype == HSPEC_F32; a.out_f32 = c.out_dtype == HSPEC_F32;
  a.status = static_cast<int*>(workspace);
  return launched(hspec::launch_adjust(a, (hipStream_t)stream));
}
