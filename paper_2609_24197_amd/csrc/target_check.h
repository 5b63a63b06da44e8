// Argument checks and workspace regions of the target-side entry points.  Host code only.
#pragma once
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
