"""Batches over the 4-bit paged cache and plain float64 forms of its operators."""
from __future__ import annotations

import math

import torch

from paper_2609_24197_amd import hspec

ST = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # a step's half of the type, relative to its binade's lower end
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def code(dtype):
    return hspec.F32 if dtype == "f32" else hspec.BF16


def power(e):
    """float64 2^e of whole numbers e, by their bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def encode(y):
    """(codes, scale bytes) [.., D] and [.., D/32] of float64 y [.., D]: the nearest magnitude by search, ties to the
    even code, under the smallest power of two with max < 7 of it (2^-126 to 2^125)."""
    b = y.reshape(*y.shape[:-1], -1, 32)
    mags = torch.tensor(MAGNITUDES, dtype=torch.float64, device=y.device)
    bad = ~(b.abs() < 2.0 ** 128 - 2.0 ** 103).all(-1)
    top = torch.where(bad, 0.0, b.abs().nan_to_num().amax(-1))
    e = torch.full_like(top, -126.0)
    for k in range(-126, 125):
        e = torch.where(top >= 7 * 2.0 ** k, float(k + 1), e)
    t = b.abs() * power(-e)[..., None]
    d = (t[..., None] - mags).abs()
    best = d.amin(-1, keepdim=True)
    near = d == best                                                     # two of them where t is half way
    even = near & (torch.arange(8, device=y.device) % 2 == 0)
    pick = torch.where(near.sum(-1, keepdim=True) > 1, even, near)
    c = pick.to(torch.uint8).argmax(-1) + 8 * torch.signbit(b)
    c = torch.where(bad[..., None], 0, c)
    return c.reshape(y.shape), torch.where(bad, 255, (e + 127).to(torch.int64))


def decode(codes, scales):
    """float64 values of codes [.., D] under scale bytes [.., D/32]."""
    mags = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float64, device=codes.device)
    s = torch.where(scales == 255, math.nan, power(scales.long() - 127))
    return mags[codes.long()] * s.repeat_interleave(32, -1)


def unpack(cache, ps, D):
    """(codes [pages, ps, Hkv, D], scale bytes [pages, ps, Hkv, D/32]) of a cache."""
    n = ps * D // 2
    by = cache[..., :n].reshape(*cache.shape[:2], ps, D // 2)
    c = torch.stack([by & 15, by >> 4], -1).reshape(*cache.shape[:2], ps, D)
    return c.transpose(1, 2), cache[..., n:].reshape(*cache.shape[:2], ps, D // 32).transpose(1, 2)


def pack(codes, scales):
    """The cache of unpack()'s two."""
    c, s = codes.transpose(1, 2).to(torch.uint8), scales.transpose(1, 2).to(torch.uint8)
    by = c[..., 0::2] | (c[..., 1::2] << 4)
    return torch.cat([by.flatten(2), s.flatten(2)], -1).contiguous()


def values(cache, ps, D):
    """float64 [pages, ps, Hkv, D]."""
    return decode(*unpack(cache, ps, D))


def batch(ctx, new, Hq, Hkv, D, ps=16, dtype="bf16", window=0, seed=0, pad_rows=2, scale=0.0, dense=None, spread=3):
    """Requests with ctx[b] cached and new[b] new tokens.  Slots that no request owns, and the tail of each last page,
    are NaN (scale byte 255).  dense: the new tokens' K and V beside the cache, "causal" or "block"; their slots in the
    cache, where pages have room, are NaN too."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, st = len(ctx), ST[dtype]
    held = [c + (0 if dense else n) for c, n in zip(ctx, new)]
    npg = [(t + ps - 1) // ps for t in held]
    pages = sum(npg) + 2
    order = torch.randperm(pages, generator=g, device="cuda").int().tolist()
    table = torch.full((B, max(max(npg), 1)), -1, dtype=torch.int32)
    caches = []
    for _ in range(2):
        c = torch.randint(0, 16, (pages, ps, Hkv, D), generator=g, device="cuda")
        s = torch.full((pages, ps, Hkv, D // 32), 255, device="cuda")
        caches.append((c, s))
    at = 0
    for b in range(B):
        ids = [order.pop() for _ in range(npg[b])]
        table[b, :npg[b]] = torch.tensor(ids, dtype=torch.int32)
        for _, s in caches:
            for i, p in enumerate(ids):
                m = min(ps, held[b] - i * ps)
                s[p, :m] = torch.randint(127 - spread, 128, (m, Hkv, D // 32), generator=g, device="cuda")
        at += npg[b]
    cu = torch.tensor([0] + new).cumsum(0).int()
    T = int(cu[-1]) + pad_rows
    draw = lambda h: torch.randn(max(T, 1), h, D, generator=g, device="cuda").to(st)  # noqa: E731
    x = dict(ctx=ctx, new=new, ps=ps, window=window, dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, T=T, q=draw(Hq), dense=dense,
             k_cache=pack(*caches[0]), v_cache=pack(*caches[1]), k_new=draw(Hkv) if dense else None,
             v_new=draw(Hkv) if dense else None, cu=cu.cuda(), lens=torch.tensor(ctx, dtype=torch.int32, device="cuda"),
             table=table.cuda(), pages=pages, max_new=max(max(new), 1),
             max_len=max(max(c + n for c, n in zip(ctx, new)), 1), scale=scale)
    x["cfg"] = hspec.chunk_cfg(B, T, x["max_new"], Hq, Hkv, D, ps, table.shape[1], pages, code(dtype), window=window,
                               scale=scale)
    return x


def attend(x, ws=None, o=None, max_len=None):
    max_len = max_len or x["max_len"]
    ws = hspec.workspace(hspec.chunk_attn_mx_workspace(x["cfg"], max_len)) if ws is None else ws
    o = torch.full_like(x["q"], 7.0) if o is None else o
    hspec.chunk_attn_mx(x["cfg"], x["q"], x["cu"], x["k_cache"], x["v_cache"], x["table"], x["lens"], max_len, o, ws,
                        k_new=x["k_new"], v_new=x["v_new"], block=x["dense"] == "block")
    return o, ws


def visible(x, L, n, i, j):
    """bool [j - i, L + n]: the keys that new tokens i .. j - 1 of a request see."""
    pos = L + torch.arange(i, j, device="cuda")[:, None]
    at = torch.arange(L + n, device="cuda")
    see = (at <= pos) | (x["dense"] == "block")
    if x["window"]:
        see = see & (at > pos - x["window"])
    return see


def keys_of(x, b, row):
    """float64 K, V [Hkv, N, D] of request b, whose first row is `row`."""
    L, n, ps, D = x["ctx"][b], x["new"][b], x["ps"], x["D"]
    held = L if x["dense"] else L + n
    ids = x["table"][b, :(held + ps - 1) // ps].long()
    out = []
    for name in "kv":
        y = values(x[name + "_cache"][ids], ps, D).reshape(-1, x["Hkv"], D)[:held]
        if x["dense"]:
            y = torch.cat([y, x[name + "_new"][row:row + n].double()])
        out.append(y.transpose(0, 1).contiguous())
    return out


def attend_ref(x):
    """(o, bound) in float64: bound is the largest error a correct kernel can have, element by element.

    Every weight may be off by half a step where it is rounded (bf16 only), by twice the score's error
    and by a few 2^-24 of its exponential; the score's error is at most D + 2 roundings of the sum of
    |q k|; summing n weights in 32 bits adds n 2^-24; the output is rounded once.  The 4-bit values are exact in
    both types."""
    Hq, Hkv, D = x["Hq"], x["Hkv"], x["D"]
    g, sc = Hq // Hkv, x["scale"] or 1 / math.sqrt(D)
    o = torch.full(x["q"].shape, 7.0, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(o)
    row = 0
    for b, (L, n) in enumerate(zip(x["ctx"], x["new"])):
        N = L + n
        K, V = keys_of(x, b, row)
        for i in range(0, n, 256):
            j = min(n, i + 256)
            see = visible(x, L, n, i, j)
            q = x["q"][row + i:row + j].double().view(j - i, Hkv, g, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D).contiguous()
            Kt = K.nan_to_num(nan=0.0, posinf=0.0, neginf=0.0).transpose(1, 2).contiguous()
            s = torch.matmul(q, Kt) * sc
            mag = torch.matmul(q.abs(), Kt.abs()) * sc
            see = see.repeat(g, 1)[None]
            p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
            p0 = torch.where(see, p, 0.0)
            vis = torch.where(see.expand_as(p0).any(1)[..., None], V, 0.0)
            big = torch.where(see, mag, 0.0).amax(-1, keepdim=True)
            back = lambda t: t.view(Hkv, g, j - i, D).permute(2, 0, 1, 3).reshape(j - i, Hq, D)  # noqa: E731
            oo, A = torch.matmul(p0, vis), torch.matmul(p0, vis.abs())
            w = 2 * (D + 2) * 2.0 ** -24 * big + (N + 32) * 2.0 ** -24 + (HALF["bf16"] if x["dtype"] == "bf16" else 0)
            o[row + i:row + j] = back(oo)
            tol[row + i:row + j] = back(w * A) + HALF[x["dtype"]] * back(oo).abs()
        row += n
    return o, tol


def check_attend(x, **kw):
    o, ws = attend(x, **kw)
    ref, tol = attend_ref(x)
    err = (o.double() - ref).abs()
    N = sum(x["new"])
    assert torch.isfinite(o[:N]).all()
    worst = ((err - tol)[:N]).max().item() if N else 0.0
    print(f"  rows {N}: max err {err[:N].max().item() if N else 0:.3e}, over bound {worst:.3e}", flush=True)
    assert worst <= 0, worst
    assert torch.equal(o[N:], torch.full_like(o[N:], 7.0))       # rows behind the last request
    return o, ws
