"""Calls of the target-side entry points that have no sound result: temperatures without a finite step, outputs over what
the call reads or writes elsewhere.  On a host without a GPU: nothing is launched."""
import ctypes as C
import math

import pytest

from paper_2609_24197_amd import hspec
from test_target_abi_cpu import FAKE, SHAPE, UNSUPPORTED, WORKSPACE, _chunk, _lib, _verify

WS = 1 << 50


@pytest.mark.parametrize("name", ["temperature", "draft_temperature"])
@pytest.mark.parametrize("value", [math.inf, 0.0, -1.0, math.nan, 1e-45])
def test_temperatures_without_a_finite_step(name, value):
    """log2(e) / T has to be positive and finite: with 0, masked logits give 0 x infinity."""
    assert _verify(**{name: value}) == SHAPE
    assert b"temperature" in _lib().hspec_last_error()


def _places(names):
    """Addresses far apart, but for those that a case moves."""
    return {n: (i + 1) << 44 for i, n in enumerate(names)}


def _refused(call, names, outs, size):
    """Each output over each other argument, by its first and by its last 16 bytes (size: bytes of an argument)."""
    L = _lib()
    base = _places(names + ["ws"])
    for out in outs + ["ws"]:
        for other in names + ["ws"]:
            if other == out:
                continue
            for at in (base[other], base[other] + (size[other] - 1) // 256 * 256, base[other] - (size[out] - 1) // 256 * 256):
                p = {**base, out: at}
                assert call(p) == UNSUPPORTED and b"lies over" in L.hspec_last_error(), (out, other, at - base[other])


def test_attention_outputs_over_other_arguments():
    L, c = _lib(), _chunk()
    need = L.hspec_chunk_attn_workspace(C.byref(c), 1000)
    names = ["q", "cu", "k", "v", "table", "lens", "o"]
    rows, cache = 68 * 32 * 128 * 2, 4096 * 16 * 8 * 128 * 2
    size = dict(q=rows, cu=20, k=cache, v=cache, table=4 * 512 * 4, lens=16, o=rows, ws=need)

    def call(p, n=need):
        return L.hspec_chunk_attn(C.byref(c), *[C.c_void_p(p[m]) for m in names[:6]], 1000, C.c_void_p(p["o"]),
                                  C.c_void_p(p["ws"]), n, None)
    _refused(call, names, ["o"], size)
    assert call(_places(names + ["ws"]), need - 1) == WORKSPACE


@pytest.mark.parametrize("code", [0, 1])
def test_append_outputs_over_other_arguments(code):
    L, c = _lib(), _chunk()
    names = ["qkv", "qw", "kw", "cu", "lens", "q", "k", "v", "table"]
    rows, cache = 68 * 32 * 128 * 2, 4096 * 16 * 8 * 128 * 2
    size = dict(qkv=68 * 48 * 128 * (4 if code else 2), qw=512, kw=512, cu=20, lens=16, q=rows, k=cache, v=cache,
                table=4 * 512 * 4, ws=256)

    def call(p):
        return L.hspec_chunk_append(C.byref(c), code, *[C.c_void_p(p[m]) for m in names], C.c_void_p(p["ws"]), 256, None)
    _refused(call, names, ["q", "k", "v"], size)


def test_verification_outputs_over_other_arguments():
    L = _lib()
    c = hspec.verify_cfg(4, 7, 32, 1000, 500, hspec.F32, 1.0, 1.0)
    need = L.hspec_verify_workspace(C.byref(c))
    names = ["target", "draft", "tok", "cu", "d2t", "t2d", "u", "gumbel", "tokens", "acc"]
    size = dict(target=32 * 4000, draft=28 * 2000, tok=112, cu=20, d2t=2000, t2d=4000, u=112, gumbel=16000, tokens=128, acc=16,
                ws=need)

    def call(p):
        return L.hspec_verify(C.byref(c), *[C.c_void_p(p[m]) for m in names], C.c_void_p(p["ws"]), need, None)
    _refused(call, names, ["tokens", "acc"], size)


def test_caches_larger_than_memory_are_compared_without_wrapping():
    c = _chunk(num_pages=2 ** 31 - 1, page_size=1 << 30, Hkv=32)
    L, names = _lib(), ["q", "cu", "k", "v", "table", "lens"]
    p = _places(names + ["o", "ws"])
    need = L.hspec_chunk_attn_workspace(C.byref(c), 1000)
    assert L.hspec_chunk_attn(C.byref(c), *[C.c_void_p(p[m]) for m in names], 1000, C.c_void_p(p["v"] + (1 << 43)),
                              C.c_void_p(p["ws"]), need, None) == UNSUPPORTED
