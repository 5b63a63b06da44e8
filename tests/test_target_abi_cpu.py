"""Refusals of the target-side entry points, on a host without a GPU: every problem the host can see returns its
status before anything touches the device."""
import ctypes as C
import os

import pytest

from paper_2609_24197_amd import hspec

FAKE = C.c_void_p(1 << 20)        # never dereferenced: validation fails first
OK, NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5


def _lib():
    if not os.path.exists(hspec.lib_path()):
        pytest.skip("libhspec.so not built")
    return hspec.lib()


def _chunk(**kw):
    c = hspec.chunk_cfg(4, 68, 17, 32, 8, 128, 16, 512, 4096)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


BAD_CHUNK = [(dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(max_new=0), SHAPE), (dict(Hq=-32), SHAPE), (dict(Hkv=0), SHAPE),
             (dict(Hkv=7), SHAPE), (dict(window=-1), SHAPE), (dict(max_pages=0), SHAPE), (dict(num_pages=0), SHAPE),
             (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
             (dict(page_size=48), UNSUPPORTED), (dict(B=40000), UNSUPPORTED), (dict(T=1 << 24), UNSUPPORTED),
             (dict(Hq=8192, T=1), UNSUPPORTED), (dict(dtype=2), DTYPE)]


OUT = C.c_void_p(1 << 40)


def _attn(c, max_len=1000, ptrs=None, ws=C.c_void_p(1 << 20), n=1 << 40, o=OUT):
    p = ptrs or [FAKE] * 6
    return _lib().hspec_chunk_attn(C.byref(c) if c else None, *p, max_len, o, ws, n, None)


def _append(c, code=1, ptrs=None, ws=C.c_void_p(1 << 20), n=1 << 40):
    p = ptrs or [FAKE] * 5 + [OUT] + [FAKE] * 3
    return _lib().hspec_chunk_append(C.byref(c) if c else None, code, *p, ws, n, None)


@pytest.mark.parametrize("kw,want", BAD_CHUNK)
def test_chunk_configs_refused(kw, want):
    assert _attn(_chunk(**kw)) == want
    assert _append(_chunk(**kw)) == want
    assert _lib().hspec_chunk_attn_workspace(C.byref(_chunk(**kw)), 1000) == 0
    assert _lib().hspec_last_error()


def test_chunk_attn_refusals():
    L, c = _lib(), _chunk()
    assert _attn(None) == NULL and L.hspec_chunk_attn_workspace(None, 10) == 0
    assert _attn(c, max_len=0) == SHAPE and L.hspec_chunk_attn_workspace(C.byref(c), 0) == 0
    assert _attn(_chunk(scale=-1.0)) == SHAPE and _attn(_chunk(scale=float("nan"))) == SHAPE
    for i in range(6):
        p = [FAKE] * 6
        p[i] = None
        assert _attn(c, ptrs=p) == NULL, i
    for i in (0, 2, 3):
        p = [FAKE] * 6
        p[i] = C.c_void_p((1 << 20) + 2)
        assert _attn(c, ptrs=p) == UNSUPPORTED, i
        assert b"aligned" in L.hspec_last_error()
    assert _attn(c, o=FAKE) == UNSUPPORTED and b"lies over" in L.hspec_last_error()
    assert _attn(c, o=C.c_void_p((1 << 20) + 68 * 32 * 128 * 2 - 16)) == UNSUPPORTED
    need = L.hspec_chunk_attn_workspace(C.byref(c), 1000)
    assert need > 0
    assert _attn(c, n=need - 1) == WORKSPACE and _attn(c, ws=None) == WORKSPACE
    assert _attn(c, ws=C.c_void_p((1 << 20) + 128)) == WORKSPACE


def test_chunk_append_refusals():
    L, c = _lib(), _chunk()
    assert _append(None) == NULL
    assert _append(c, code=3) == DTYPE
    assert _append(_chunk(rope_theta=0.0)) == SHAPE and _append(_chunk(rope_theta=float("nan"))) == SHAPE
    for i in range(9):                                       # (1 and 2, the gains, only together)
        p = [FAKE] * 9
        p[i] = None
        assert _append(c, ptrs=p) == NULL, i
    for i in (0, 5, 6, 7):
        p = [FAKE] * 9
        p[i] = C.c_void_p((1 << 20) + 8)
        assert _append(c, ptrs=p) == UNSUPPORTED, i
    assert _append(c, ptrs=[FAKE] * 9) == UNSUPPORTED and b"lies over" in L.hspec_last_error()
    assert _append(c, n=8) == WORKSPACE
    assert L.hspec_chunk_append_workspace(C.byref(c)) >= 256


def _verify(ptrs=None, n=1 << 40, ws=C.c_void_p(1 << 20), cfg=True, **kw):
    c = hspec.verify_cfg(4, 7, 32, 1000, 500, hspec.F32, 1.0, 1.0)
    for k, v in kw.items():
        setattr(c, k, v)
    names = ["target", "draft", "tok", "cu", "d2t", "t2d", "u", "gumbel", "tokens", "acc"]
    p = {m: FAKE for m in names} | (ptrs or {})
    return _lib().hspec_verify(C.byref(c) if cfg else None, *[p[m] for m in names], ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(cfg=False), NULL), (dict(B=0), SHAPE), (dict(k=0), SHAPE), (dict(rows=0), SHAPE), (dict(vocab=0), SHAPE),
    (dict(draft_vocab=0), SHAPE), (dict(draft_vocab=1001), SHAPE), (dict(vocab=1 << 29), UNSUPPORTED),
    (dict(B=40000), UNSUPPORTED), (dict(k=5000), UNSUPPORTED), (dict(rows=1 << 23), UNSUPPORTED), (dict(dtype=9), DTYPE),
    (dict(temperature=0.0), SHAPE), (dict(temperature=-1.0), SHAPE), (dict(temperature=float("nan")), SHAPE),
    (dict(temperature=1e-45), SHAPE), (dict(draft_temperature=0.0), SHAPE),
    (dict(ptrs=dict(target=None)), NULL), (dict(ptrs=dict(tok=None)), NULL), (dict(ptrs=dict(tokens=None)), NULL),
    (dict(ptrs=dict(acc=None)), NULL), (dict(ptrs=dict(u=None)), NULL), (dict(ptrs=dict(gumbel=None)), NULL),
    (dict(ptrs=dict(u=None, gumbel=None)), UNSUPPORTED), (dict(ptrs=dict(d2t=None)), NULL), (dict(ptrs=dict(t2d=None)), NULL),
    (dict(ptrs=dict(cu=None), rows=31), SHAPE), (dict(n=16), WORKSPACE), (dict(ws=None), WORKSPACE)])
def test_verify_refusals(kw, want):
    assert _verify(**kw) == want
    assert _lib().hspec_last_error()


def test_tokens_over_drafts_are_refused():
    far = C.c_void_p(FAKE.value + (1 << 24))
    for tok, tokens in ((FAKE, FAKE), (FAKE, C.c_void_p(FAKE.value + 4 * 7 * 4 - 4)), (C.c_void_p(FAKE.value + 4 * 8 * 4 - 4), FAKE)):
        assert _verify(ptrs=dict(tok=tok, tokens=tokens, acc=far)) == UNSUPPORTED
        assert b"lies over" in _lib().hspec_last_error()


def test_workspace_of_a_bad_verification_is_zero():
    c = hspec.verify_cfg(4, 7, 32, 1000, 2000)
    assert _lib().hspec_verify_workspace(C.byref(c)) == 0


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 3)                                    # (a host tensor: device -1)
    assert hspec._arg("x", x, torch.float32, (2, 3), -1) == x.data_ptr()
    assert hspec._arg("x", None, torch.float32, (2, 3), -1) is None
    for bad in (x.int(), x[:1], x.t(), torch.zeros(2, 6)[:, ::2]):
        with pytest.raises(ValueError, match="x: expected"):
            hspec._arg("x", bad, torch.float32, (2, 3), -1)
    with pytest.raises(ValueError, match="on the current device"):
        hspec._arg("x", x, torch.float32, (2, 3), 0)
    with pytest.raises(ValueError, match="ws"):
        hspec._run(None, 0, torch.zeros(8, dtype=torch.uint8))
