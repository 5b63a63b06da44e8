"""Refusals of the 4-bit cache's entry points and of the logits' adjustment, on a host without a GPU: every problem the
host can see returns its status before anything touches the device."""
import ctypes as C
import os

import pytest

from paper_2609_24197_amd import hspec
from test_target_abi_cpu import BAD_CHUNK, DTYPE, FAKE, NULL, OUT, SHAPE, UNSUPPORTED, WORKSPACE, _chunk

MIS = C.c_void_p((1 << 20) + 8)


def _lib():
    if not os.path.exists(hspec.lib_path()):
        pytest.skip("libhspec.so not built")
    return hspec.lib()


def far(i):
    """Places far from one another and from FAKE."""
    return C.c_void_p((i + 1) << 42)


WS = far(0)
# arguments that a call of each takes: inputs at FAKE, outputs apart
APPEND = [FAKE] * 5 + [far(1), far(2), far(3), FAKE]
READ = [FAKE] * 5 + [far(1), far(2)]
ATTN = [FAKE, FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 1000, far(1)]


def _append(c, args=None, ws=WS, n=1 << 40, dtype=1):
    return _lib().hspec_chunk_append_mx(C.byref(c) if c else None, dtype, *(args or APPEND), ws, n, None)


def _read(c, args=None, ws=WS, n=1 << 40):
    return _lib().hspec_chunk_read_mx(C.byref(c) if c else None, *(args or READ), ws, n, None)


def _attn(c, args=None, ws=WS, n=1 << 40):
    return _lib().hspec_chunk_attn_mx(C.byref(c) if c else None, *(args or ATTN), ws, n, None)


CALLS = [(_append, APPEND), (_read, READ), (_attn, ATTN)]


@pytest.mark.parametrize("kw,want", BAD_CHUNK)
def test_configs_refused(kw, want):
    for call, _ in CALLS:
        assert call(_chunk(**kw)) == want
    assert _lib().hspec_chunk_attn_mx_workspace(C.byref(_chunk(**kw)), 1000) == 0
    assert _lib().hspec_mx_cache_bytes(C.byref(_chunk(**kw))) == 0
    assert _lib().hspec_last_error()


def swap(args, i, v):
    return args[:i] + [v] + args[i + 1:]


def test_pointers_refused():
    c = _chunk()
    for call, args in CALLS:
        assert call(None) == NULL
        for i, a in enumerate(args):
            if isinstance(a, int):
                continue
            both = call is _attn and i in (2, 3) or call is _append and i in (1, 2)     # NULL together only
            assert call(c, swap(args, i, None)) == NULL, (call, i, both)
        assert call(c, ws=None) == WORKSPACE
        assert call(c, ws=C.c_void_p(WS.value + 8)) == WORKSPACE
        assert call(c, n=64) == WORKSPACE
    # tensors that are read 16 bytes at a time (not the norms' gains and the batch's whole numbers)
    for call, args, tensors in ((_append, APPEND, (0, 5, 6, 7)), (_read, READ, (2, 3, 5, 6)), (_attn, ATTN, (0, 2, 3, 5, 6, 10))):
        for i in tensors:
            at = args[i].value + 8
            assert call(c, swap(args, i, C.c_void_p(at))) == UNSUPPORTED, (call, i)


def test_outputs_over_inputs_refused():
    c = _chunk()
    for call, args, outs in ((_append, APPEND, (5, 6, 7)), (_read, READ, (5, 6)), (_attn, ATTN, (10,))):
        for i in outs:
            assert call(c, swap(args, i, FAKE)) == UNSUPPORTED, (call, i)
            assert call(c, ws=args[i]) == UNSUPPORTED, (call, i)
        for i in outs[1:]:
            assert call(c, swap(args, i, args[outs[0]])) == UNSUPPORTED, (call, i)
        assert b"lies over" in _lib().hspec_last_error()


def test_settings_refused():
    c = _chunk()
    assert _append(c, dtype=5) == DTYPE
    c.rope_theta = 0.0
    assert _append(c) == SHAPE
    c = _chunk()
    assert _attn(c, swap(ATTN, 9, 0)) == SHAPE
    assert _lib().hspec_chunk_attn_mx_workspace(C.byref(c), 0) == 0
    assert _attn(_chunk(scale=-1.0)) == SHAPE and _attn(_chunk(scale=float("nan"))) == SHAPE
    assert _attn(c, swap(ATTN, 4, 2)) == UNSUPPORTED
    none = swap(swap(ATTN, 2, None), 3, None)
    assert _attn(c, swap(none, 4, 1)) == NULL
    assert _attn(_chunk(window=16), swap(ATTN, 4, 1)) == UNSUPPORTED          # max_new 17
    assert _lib().hspec_mx_cache_bytes(C.byref(c)) == 4096 * 8 * 16 * 68


LOGITS, CU, DRAFTS, D2T, HIST, LENS, PROMPT, REP, FREQ, PRES, IDS, BIAS, MASK, ROWS, AT_OUT = range(15)


def _adjust_cfg(**kw):
    c = hspec.adjust_cfg(4, 3, 16, 1000, 500, 64, 5, 16)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def _adjust(c=None, ws=WS, n=256, **kw):
    args = [far(2)] + [FAKE] * 13 + [far(1)]
    for i, v in kw.pop("at", {}).items():
        args[i] = v
    c = _adjust_cfg(**kw) if c is None else c
    return _lib().hspec_adjust_logits(C.byref(c) if c else None, *args, ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), SHAPE), (dict(k=-1), SHAPE), (dict(rows=0), SHAPE), (dict(vocab=0), SHAPE), (dict(draft_vocab=-1), SHAPE),
    (dict(max_hist=-1), SHAPE), (dict(n_bias=-1), SHAPE), (dict(masks=-1), SHAPE), (dict(dtype=2), DTYPE),
    (dict(out_dtype=-1), DTYPE), (dict(vocab=1 << 20), UNSUPPORTED), (dict(draft_vocab=1 << 20), UNSUPPORTED),
    (dict(B=40000), UNSUPPORTED), (dict(k=5000), UNSUPPORTED), (dict(B=32767, k=4096), UNSUPPORTED),
    (dict(rows=1 << 23), UNSUPPORTED), (dict(max_hist=(1 << 24) + 1), UNSUPPORTED), (dict(n_bias=(1 << 20) + 1), UNSUPPORTED),
    (dict(masks=(1 << 22) + 1), UNSUPPORTED)])
def test_adjust_configs_refused(kw, want):
    assert _adjust(**kw) == want
    assert _lib().hspec_adjust_logits_workspace(C.byref(_adjust_cfg(**kw))) == 0


def test_adjust_arguments_refused():
    L = _lib()
    assert L.hspec_adjust_logits(None, *[FAKE] * 15, WS, 256, None) == NULL
    for i in (LOGITS, HIST, LENS, IDS, BIAS, MASK, AT_OUT):
        assert _adjust(at={i: None}) == NULL, i
    assert _adjust(max_hist=0) == NULL and _adjust(n_bias=0) == NULL and _adjust(masks=0) == NULL
    assert _adjust(at={HIST: None, LENS: None}, max_hist=0) == NULL        # the prompt's lengths are left
    assert _adjust(at={MASK: None}, masks=0) == NULL                       # the rows' lines are left
    assert _adjust(at={ROWS: None}, masks=15) == SHAPE
    assert _adjust(at={CU: None}, rows=17, masks=17) == SHAPE
    assert _adjust(k=0) == SHAPE and _adjust(draft_vocab=0) == SHAPE
    assert _adjust(ws=None) == WORKSPACE and _adjust(n=255) == WORKSPACE
    assert _adjust(ws=C.c_void_p(WS.value + 16)) == WORKSPACE
    assert _adjust(at={LOGITS: C.c_void_p((1 << 43) + 1)}) == UNSUPPORTED
    assert _adjust(at={AT_OUT: C.c_void_p((1 << 43) + 2)}, out_dtype=1) == UNSUPPORTED
    assert _adjust(at={AT_OUT: far(2)}, out_dtype=1) == UNSUPPORTED        # in place, another type
    assert _adjust(at={AT_OUT: C.c_void_p(far(2).value + 2000)}) == UNSUPPORTED
    for i in range(1, 14):
        assert _adjust(at={AT_OUT: FAKE}) == UNSUPPORTED
    assert _adjust(ws=far(1)) == UNSUPPORTED and _adjust(ws=far(2)) == UNSUPPORTED
