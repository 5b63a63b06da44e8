"""Outputs and workspaces over the inputs of the 4-bit cache's calls and of the logits' adjustment, one input at a time, on a
host without a GPU.  Every argument has a place of its own, so that each refusal is that input's alone."""
import ctypes as C

import pytest
import torch

from paper_2609_24197_amd import hspec
from test_mx_abi_cpu import _adjust_cfg, _append, _attn, _lib, _read, far
from test_target_abi_cpu import OK, UNSUPPORTED, _chunk

WS = far(0)
NAMES = {
    "append": ["qkv", "q_norm_w", "k_norm_w", "cu_new", "ctx_lens", "q", "k_cache", "v_cache", "page_table"],
    "read": ["cu_new", "ctx_lens", "k_cache", "v_cache", "page_table", "k", "v"],
    "attn": ["q", "cu_new", "k_new", "v_new", 0, "k_cache", "v_cache", "page_table", "ctx_lens", 1000, "o"],
    "adjust": ["logits", "cu_rows", "draft_tokens", "d2t", "history", "hist_lens", "prompt_lens", "repetition", "frequency",
               "presence", "bias_ids", "bias", "mask", "mask_rows", "out"],
}
OUTS = {"append": ["q", "k_cache", "v_cache"], "read": ["k", "v"], "attn": ["o"], "adjust": ["out"]}
# bytes of the last element of each argument, from its start: the 4 requests, 68 rows, 32 and 8 heads of 128, pages of 16 and
# the adjustment's 16 rows of 1000 that the configurations below have
BYTES = {"qkv": 68 * 48 * 128 * 4, "q_norm_w": 512, "k_norm_w": 512, "cu_new": 20, "ctx_lens": 16, "q": 68 * 32 * 128 * 2,
         "k_cache": 4096 * 8 * 16 * 68, "v_cache": 4096 * 8 * 16 * 68, "page_table": 4 * 512 * 4, "k": 68 * 8 * 128 * 2,
         "v": 68 * 8 * 128 * 2, "k_new": 68 * 8 * 128 * 2, "v_new": 68 * 8 * 128 * 2, "o": 68 * 32 * 128 * 2,
         "logits": 16 * 1000 * 2, "out": 16 * 1000 * 2, "cu_rows": 20, "draft_tokens": 48, "d2t": 2000, "history": 1024,
         "hist_lens": 16, "prompt_lens": 16, "repetition": 16, "frequency": 16, "presence": 16, "bias_ids": 80, "bias": 80,
         "mask": 16 * 32 * 4, "mask_rows": 64}


def call(op, places, ws=WS):
    args = [places[n] if isinstance(n, str) else n for n in NAMES[op]]
    if op == "adjust":
        return _lib().hspec_adjust_logits(C.byref(_adjust_cfg()), *args, ws, 256, None)
    return {"append": _append, "read": _read, "attn": _attn}[op](_chunk(), args, ws=ws)


def places(op):
    return {n: far(i + 1) for i, n in enumerate(NAMES[op]) if isinstance(n, str)}


PAIRS = [(op, out, n) for op in NAMES for out in OUTS[op] + ["workspace"] for n in NAMES[op]
         if isinstance(n, str) and n != out and (op, out, n) != ("adjust", "out", "logits")]


@pytest.mark.parametrize("op,out,over", PAIRS)
def test_each_input_refused(op, out, over):
    p = places(op)
    assert all(v < 1 << 42 for v in BYTES.values())
    # over the argument's start, and over what its last 256 bytes hold (a workspace is 256-byte aligned)
    for at in (0, max(BYTES[over] - 1, 0) // 256 * 256):
        place = C.c_void_p(p[over].value + at)
        if out == "workspace":
            s = call(op, p, ws=place)
        else:
            s = call(op, dict(p, **{out: place}))
        assert s == UNSUPPORTED, (op, out, over, at)
        assert b"lies over" in _lib().hspec_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call with these places must not reach a GPU")
@pytest.mark.parametrize("op", sorted(NAMES))
def test_places_apart_are_not_refused(op):
    """The refusals above are of the overlap: without one the call gets as far as the launch, which a host without a GPU fails."""
    s = call(op, places(op))
    assert hspec.STATUS.get(s) == hspec.STATUS[6] and s not in (OK, UNSUPPORTED)
