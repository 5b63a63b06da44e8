"""ctypes binding of libhspec.so (the C ABI declared in include/hspec.h).

Argument marshalling only: torch tensors provide device memory and the current HIP stream;
every step of the drafting path runs in the library's kernels.  Importing this module does
not touch the GPU; ``lib()`` loads the shared library and raises if it is missing, so a
missing build can never fall back to anything else.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import inputs as I

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhspec.so")
_lib = None

BF16, F32 = 0, 1
BLOCK_CAUSAL = 1
ATTN_PRECISE_IO = 2
CHUNK_BLOCK = 1
W_DS_PACKED = 1
MAMBA_PRECISE_IO = 2
DEV_BAD_PAGE, DEV_BAD_CTX_LEN, DEV_BAD_TOKEN, DEV_NONFINITE, DEV_BAD_ROWS = 1, 2, 4, 8, 16
STATUS = {0: "HSPEC_OK", 1: "HSPEC_ERR_NULL", 2: "HSPEC_ERR_SHAPE", 3: "HSPEC_ERR_DTYPE",
          4: "HSPEC_ERR_UNSUPPORTED", 5: "HSPEC_ERR_WORKSPACE", 6: "HSPEC_ERR_LAUNCH"}


class MambaCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "k", "d_model", "d_h", "r", "H", "P", "N", "G", "chunk", "conv_w")] + [
        ("flags", C.c_uint), ("dtype", C.c_int), ("eps", C.c_float)]


class MambaW(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("W_r", "W_dS", "W_in", "conv_w", "conv_b", "dt_bias", "A_log", "D",
                                           "gnorm_w", "W_out")]


class AttnCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "k", "d_model", "Hq", "Hkv", "D", "page_size", "max_pages",
                                        "num_pages", "window", "split_tokens")] + [
        ("flags", C.c_uint), ("dtype", C.c_int), ("eps", C.c_float), ("scale", C.c_float),
        ("rope_theta", C.c_double), ("Hkv_cache", C.c_int), ("kv_heads", C.POINTER(C.c_int32))]


class AttnW(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("W_q", "W_k", "W_v", "W_o", "q_norm_w", "k_norm_w")]


class LayerW(C.Structure):
    _fields_ = [("mamba", C.POINTER(MambaW)), ("norm1_w", C.c_void_p), ("attn", C.POINTER(AttnW)),
                ("norm2_w", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("norm3_w", C.c_void_p),
                ("W_gate", C.c_void_p), ("W_up", C.c_void_p), ("W_down", C.c_void_p)]


class HeadCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "k", "d_model", "vocab", "rank")] + [
        ("eps", C.c_float), ("temperature", C.c_float)]


class HeadW(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("norm_f_w", "W_lm", "E_M", "U_M")]


class ChunkCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "T", "max_new", "Hq", "Hkv", "D", "page_size", "max_pages", "num_pages",
                                        "window")] + [
        ("dtype", C.c_int), ("eps", C.c_float), ("scale", C.c_float), ("rope_theta", C.c_double)]


class VerifyCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "k", "rows", "vocab", "draft_vocab")] + [
        ("dtype", C.c_int), ("temperature", C.c_float), ("draft_temperature", C.c_float)]


class AdjustCfg(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "k", "rows", "vocab", "draft_vocab", "max_hist", "n_bias", "masks", "dtype",
                                        "out_dtype")]


class HspecError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


EXPORTS = {
    "hspec_mamba_block_scan": (C.c_int, [C.POINTER(MambaCfg), C.POINTER(MambaW), C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hspec_mamba_block_scan_workspace": (C.c_size_t, [C.POINTER(MambaCfg)]),
    "hspec_target_kv_block_attn": (C.c_int, [C.POINTER(AttnCfg), C.POINTER(AttnW), C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                             C.c_size_t, C.c_void_p]),
    "hspec_target_kv_block_attn_workspace": (C.c_size_t, [C.POINTER(AttnCfg), C.c_int]),
    "hspec_draft_step": (C.c_int, [C.POINTER(MambaCfg), C.POINTER(MambaW), C.c_void_p, C.POINTER(AttnCfg),
                                   C.POINTER(AttnW), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hspec_draft_step_workspace": (C.c_size_t, [C.POINTER(MambaCfg), C.POINTER(AttnCfg), C.c_int]),
    "hspec_state_init": (C.c_int, [C.POINTER(MambaCfg), C.POINTER(MambaW), C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_size_t, C.c_void_p]),
    "hspec_state_init_workspace": (C.c_size_t, [C.POINTER(MambaCfg)]),
    "hspec_ssd_scan": (C.c_int, [C.c_int] * 7 + [C.c_int] + [C.c_void_p] * 9 + [C.c_void_p, C.c_size_t, C.c_void_p]),
    "hspec_ssd_scan_workspace": (C.c_size_t, [C.c_int] * 7),
    "hspec_paged_attn": (C.c_int, [C.POINTER(AttnCfg)] + [C.c_void_p] * 7 + [C.c_int, C.c_void_p, C.c_void_p,
                                                                          C.c_size_t, C.c_void_p]),
    "hspec_paged_attn_static": (C.c_int, [C.POINTER(AttnCfg), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                          C.c_void_p]),
    "hspec_paged_attn_workspace": (C.c_size_t, [C.POINTER(AttnCfg), C.c_int]),
    "hspec_paged_attn_phase": (C.c_int, [C.POINTER(AttnCfg)] + [C.c_void_p] * 7 + [C.c_int, C.c_void_p, C.c_void_p,
                                                                                C.c_size_t, C.c_uint, C.c_void_p]),
    "hspec_gather_slots": (C.c_int, [C.c_int] * 4 + [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                                      C.c_void_p]),
    "hspec_linear": (C.c_int, [C.c_int] * 4 + [C.c_void_p] * 5 + [C.c_size_t, C.c_void_p]),
    "hspec_linear_workspace": (C.c_size_t, [C.c_int] * 4),
    "hspec_drafter_forward": (C.c_int, [C.POINTER(MambaCfg), C.POINTER(AttnCfg), C.c_int, C.c_int, C.c_void_p,
                                        C.c_void_p, C.POINTER(LayerW)] + [C.c_void_p] * 4 + [C.c_int, C.c_void_p,
                                                                                             C.c_void_p, C.c_size_t,
                                                                                             C.c_void_p]),
    "hspec_drafter_forward_workspace": (C.c_size_t, [C.POINTER(MambaCfg), C.POINTER(AttnCfg), C.c_int, C.c_int]),
    "hspec_kv_inject": (C.c_int, [C.POINTER(AttnCfg), C.c_int, C.c_int, C.c_void_p, C.c_void_p] +
                        [C.POINTER(C.c_void_p)] * 5 + [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hspec_kv_inject_workspace": (C.c_size_t, [C.POINTER(AttnCfg), C.c_int]),
    "hspec_draft_head": (C.c_int, [C.POINTER(HeadCfg), C.POINTER(HeadW)] + [C.c_void_p] * 7 + [C.c_size_t,
                                                                                          C.c_void_p]),
    "hspec_draft_head_workspace": (C.c_size_t, [C.POINTER(HeadCfg)]),
    "hspec_chunk_append": (C.c_int, [C.POINTER(ChunkCfg), C.c_int] + [C.c_void_p] * 10 + [C.c_size_t, C.c_void_p]),
    "hspec_chunk_append_workspace": (C.c_size_t, [C.POINTER(ChunkCfg)]),
    "hspec_chunk_attn": (C.c_int, [C.POINTER(ChunkCfg)] + [C.c_void_p] * 6 + [C.c_int, C.c_void_p, C.c_void_p, C.c_size_t,
                                                                          C.c_void_p]),
    "hspec_chunk_attn_workspace": (C.c_size_t, [C.POINTER(ChunkCfg), C.c_int]),
    "hspec_verify": (C.c_int, [C.POINTER(VerifyCfg)] + [C.c_void_p] * 11 + [C.c_size_t, C.c_void_p]),
    "hspec_verify_workspace": (C.c_size_t, [C.POINTER(VerifyCfg)]),
    "hspec_mx_cache_bytes": (C.c_size_t, [C.POINTER(ChunkCfg)]),
    "hspec_chunk_append_mx": (C.c_int, [C.POINTER(ChunkCfg), C.c_int] + [C.c_void_p] * 10 + [C.c_size_t, C.c_void_p]),
    "hspec_chunk_append_mx_workspace": (C.c_size_t, [C.POINTER(ChunkCfg)]),
    "hspec_chunk_read_mx": (C.c_int, [C.POINTER(ChunkCfg)] + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]),
    "hspec_chunk_read_mx_workspace": (C.c_size_t, [C.POINTER(ChunkCfg)]),
    "hspec_chunk_attn_mx": (C.c_int, [C.POINTER(ChunkCfg)] + [C.c_void_p] * 4 + [C.c_uint] + [C.c_void_p] * 4 +
                            [C.c_int, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hspec_chunk_attn_mx_workspace": (C.c_size_t, [C.POINTER(ChunkCfg), C.c_int]),
    "hspec_adjust_logits": (C.c_int, [C.POINTER(AdjustCfg)] + [C.c_void_p] * 16 + [C.c_size_t, C.c_void_p]),
    "hspec_adjust_logits_workspace": (C.c_size_t, [C.POINTER(AdjustCfg)]),
    "hspec_pack_w_ds_bytes": (C.c_size_t, [C.c_int, C.c_int]),
    "hspec_pack_w_ds": (C.c_int, [C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hspec_read_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.c_void_p]),
    "hspec_status_string": (C.c_char_p, [C.c_int]),
    "hspec_last_error": (C.c_char_p, []),
}


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libhspec.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with paper_2609_24197_amd.build")
        L = C.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise HspecError(status, lib().hspec_last_error().decode())


# --------------------------------------------------------------------------- torch side

def _torch():
    import torch
    return torch


def stream_ptr():
    return C.c_void_p(_torch().cuda.current_stream().cuda_stream)


def ptr(t):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "expected a contiguous device tensor"
    return C.c_void_p(t.data_ptr())


def to_device(a: np.ndarray, dev="cuda"):
    """Storage array (uint16 bf16 bits, float32, int32) -> device tensor of the same bits."""
    torch = _torch()
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).to(dev)
    return torch.from_numpy(a).to(dev)


def workspace(nbytes: int, dev="cuda"):
    torch = _torch()
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=dev)


def dtype_code(cfg: I.StepConfig) -> int:
    return F32 if cfg.dtype == "f32" else BF16


def mamba_cfg(cfg: I.StepConfig, W: dict | None = None) -> MambaCfg:
    """The Mamba config; W_DS_PACKED is set when W carries "W_dS_packed" (see pack_w_ds), and
    MAMBA_PRECISE_IO with the config's precise_io."""
    flags = W_DS_PACKED if W is not None and W.get("W_dS_packed") is not None else 0
    flags |= MAMBA_PRECISE_IO if cfg.precise_io else 0
    return MambaCfg(cfg.B, cfg.k, cfg.d_model, cfg.d_h, cfg.rank, cfg.H, cfg.P, cfg.N, cfg.G, cfg.chunk,
                    cfg.conv_w, flags, dtype_code(cfg), cfg.eps)


def attn_cfg(cfg: I.StepConfig, max_pages: int, num_pages: int) -> AttnCfg:
    c = AttnCfg(cfg.B, cfg.k, cfg.d_model, cfg.Hq, cfg.Hkv, cfg.D, cfg.page_size, max_pages, num_pages,
                cfg.window, cfg.split_tokens,
                (BLOCK_CAUSAL if cfg.block_causal else 0) | (ATTN_PRECISE_IO if cfg.precise_io else 0), dtype_code(cfg),
                cfg.eps, 0.0, cfg.rope_theta, cfg.Hkv_target, None)
    if cfg.kv_heads:   # partial target-KV-head reuse: the array lives as long as the config
        c._kv_heads = (C.c_int32 * len(cfg.kv_heads))(*cfg.kv_heads)
        c.kv_heads = C.cast(c._kv_heads, C.POINTER(C.c_int32))
    return c


def mamba_w(W: dict) -> MambaW:
    """Weight pointers; a "W_dS_packed" entry replaces W_dS (pair it with mamba_cfg(cfg, W))."""
    names = ("W_r", "W_dS", "W_in", "conv_w", "conv_b", "dt_bias", "A_log", "D", "gnorm_w", "W_out")
    return MambaW(*(ptr(W.get("W_dS_packed", W.get("W_dS")) if n == "W_dS" else W.get(n)) for n in names))


def pack_w_ds(W_dS, d_S: int, r: int):
    """The packed copy of a bf16 W_dS [d_S, r] device tensor (hspec_pack_w_ds), as a new tensor."""
    import torch
    nbytes = lib().hspec_pack_w_ds_bytes(int(d_S), int(r))
    if nbytes == 0:
        raise HspecError(4, "W_dS shape cannot be packed")
    out = torch.empty(nbytes // 2, dtype=torch.bfloat16, device=W_dS.device)
    _check(lib().hspec_pack_w_ds(int(d_S), int(r), ptr(W_dS), ptr(out), stream_ptr()))
    return out


def attn_w(W: dict) -> AttnW:
    return AttnW(*(ptr(W.get(n)) for n in ("W_q", "W_k", "W_v", "W_o", "q_norm_w", "k_norm_w")))


def read_status(ws) -> int:
    v = C.c_int32(0)
    _check(lib().hspec_read_status(ptr(ws), C.byref(v), stream_ptr()))
    return int(v.value)


# ------------------------------------------------------------------------ entry points

def draft_step_workspace(cfg, max_pages, num_pages, max_ctx_len) -> int:
    mc, ac = mamba_cfg(cfg), attn_cfg(cfg, max_pages, num_pages)
    return lib().hspec_draft_step_workspace(C.byref(mc), C.byref(ac), int(max_ctx_len))


def draft_step(cfg, W: dict, X: dict, out, ws, max_ctx_len: int):
    """out [B, k, d_model] fp32 = one drafting step (see hspec_draft_step)."""
    mc = mamba_cfg(cfg, W)
    ac = attn_cfg(cfg, X["page_table"].shape[1], X["k_cache"].shape[0])
    mw, aw = mamba_w(W), attn_w(W)
    _check(lib().hspec_draft_step(C.byref(mc), C.byref(mw), ptr(W["norm1_w"]), C.byref(ac), C.byref(aw),
                                  ptr(W["norm2_w"]), ptr(X["h_last"]), ptr(X["block_emb"]), ptr(X["k_cache"]),
                                  ptr(X["v_cache"]), ptr(X["page_table"]), ptr(X["ctx_lens"]), int(max_ctx_len),
                                  ptr(out), ptr(ws), ws.numel(), stream_ptr()))


def mamba_block_scan_workspace(cfg) -> int:
    mc = mamba_cfg(cfg)
    return lib().hspec_mamba_block_scan_workspace(C.byref(mc))


def mamba_block_scan(cfg, W, h_last, u, out, ws, S_final=None):
    mc, mw = mamba_cfg(cfg, W), mamba_w(W)
    _check(lib().hspec_mamba_block_scan(C.byref(mc), C.byref(mw), ptr(h_last), ptr(u), ptr(out), ptr(S_final),
                                        ptr(ws), ws.numel(), stream_ptr()))


def target_kv_block_attn_workspace(cfg, max_pages, num_pages, max_ctx_len) -> int:
    ac = attn_cfg(cfg, max_pages, num_pages)
    return lib().hspec_target_kv_block_attn_workspace(C.byref(ac), int(max_ctx_len))


def target_kv_block_attn(cfg, W, x, X, out, ws, max_ctx_len):
    ac = attn_cfg(cfg, X["page_table"].shape[1], X["k_cache"].shape[0])
    aw = attn_w(W)
    _check(lib().hspec_target_kv_block_attn(C.byref(ac), C.byref(aw), ptr(x), ptr(X["k_cache"]), ptr(X["v_cache"]),
                                            ptr(X["page_table"]), ptr(X["ctx_lens"]), int(max_ctx_len), ptr(out),
                                            ptr(ws), ws.numel(), stream_ptr()))


def state_init_workspace(cfg) -> int:
    mc = mamba_cfg(cfg)
    return lib().hspec_state_init_workspace(C.byref(mc))


def state_init(cfg, W, h_last, S0, ws):
    mc, mw = mamba_cfg(cfg, W), mamba_w(W)
    _check(lib().hspec_state_init(C.byref(mc), C.byref(mw), ptr(h_last), ptr(S0), ptr(ws), ws.numel(),
                                  stream_ptr()))


def ssd_scan_workspace(B, T, H, P, N, G, dtype) -> int:
    return lib().hspec_ssd_scan_workspace(B, T, H, P, N, G, dtype)


def ssd_scan(B, T, H, P, N, G, chunk, dtype, x, dt, A, Bm, Cm, Dskip, S0, y, S_final, ws):
    _check(lib().hspec_ssd_scan(B, T, H, P, N, G, chunk, dtype, ptr(x), ptr(dt), ptr(A), ptr(Bm), ptr(Cm),
                                ptr(Dskip), ptr(S0), ptr(y), ptr(S_final), ptr(ws), ws.numel(), stream_ptr()))


def paged_attn_workspace(cfg, max_pages, num_pages, max_ctx_len) -> int:
    ac = attn_cfg(cfg, max_pages, num_pages)
    return lib().hspec_paged_attn_workspace(C.byref(ac), int(max_ctx_len))


PHASE_WORKLIST, PHASE_SWEEP, PHASE_REDUCE = 1, 2, 4


def paged_attn(cfg, X, o, ws, max_ctx_len, acfg: AttnCfg | None = None, phases: int | None = None):
    """All of the attention core, or (phases: OR of PHASE_*) some of its launches in order."""
    ac = acfg or attn_cfg(cfg, X["page_table"].shape[1], X["k_cache"].shape[0])
    args = (C.byref(ac), ptr(X["q"]), ptr(X["k_blk"]), ptr(X["v_blk"]), ptr(X["k_cache"]), ptr(X["v_cache"]),
            ptr(X["page_table"]), ptr(X["ctx_lens"]), int(max_ctx_len), ptr(o), ptr(ws), ws.numel())
    if phases is None:
        _check(lib().hspec_paged_attn(*args, stream_ptr()))
    else:
        _check(lib().hspec_paged_attn_phase(*args, int(phases), stream_ptr()))


STATIC_WS_BYTES = 64 << 20   # HSPEC_STATIC_WS_BYTES


def paged_attn_static(cfg, X, o, max_ctx_len, status=None, acfg: AttnCfg | None = None):
    """The attention core on the library's fixed device array (no workspace argument)."""
    ac = acfg or attn_cfg(cfg, X["page_table"].shape[1], X["k_cache"].shape[0])
    _check(lib().hspec_paged_attn_static(C.byref(ac), ptr(X["q"]), ptr(X["k_blk"]), ptr(X["v_blk"]),
                                         ptr(X["k_cache"]), ptr(X["v_cache"]), ptr(X["page_table"]),
                                         ptr(X["ctx_lens"]), int(max_ctx_len), ptr(o), ptr(status), stream_ptr()))


def gather_slots(page_table, ctx_lens, page_size, num_pages, max_ctx_len, slots, status=None):
    B, max_pages = page_table.shape
    _check(lib().hspec_gather_slots(B, max_pages, page_size, num_pages, ptr(page_table), ptr(ctx_lens),
                                    int(max_ctx_len), ptr(slots), ptr(status), stream_ptr()))


def linear_workspace(dtype, M, N, K) -> int:
    return lib().hspec_linear_workspace(dtype, M, N, K)


def linear(dtype, A, W, C_out, ws, R=None):
    M, K = A.shape
    N = W.shape[0]
    _check(lib().hspec_linear(dtype, M, N, K, ptr(A), ptr(W), ptr(R), ptr(C_out), ptr(ws), ws.numel(),
                              stream_ptr()))


def head_cfg(cfg, vocab: int, rank: int, temperature: float = 1.0) -> HeadCfg:
    return HeadCfg(cfg.B, cfg.k, cfg.d_model, int(vocab), int(rank), cfg.eps, float(temperature))


def draft_head_workspace(hc: HeadCfg) -> int:
    return lib().hspec_draft_head_workspace(C.byref(hc))


def draft_head(hc: HeadCfg, W: dict, hidden, prev_tok, tokens, ws, logits=None, gumbel=None, forced=None):
    """tokens [B, k] int32 (and the corrected logits [B, k, V] if given) = hspec_draft_head."""
    hw = HeadW(*(ptr(W[n]) for n in ("norm_f_w", "W_lm", "E_M", "U_M")))
    _check(lib().hspec_draft_head(C.byref(hc), C.byref(hw), ptr(hidden), ptr(prev_tok), ptr(gumbel), ptr(forced),
                                  ptr(tokens), ptr(logits), ptr(ws), ws.numel(), stream_ptr()))


def drafter_forward_workspace(cfg, max_pages, num_pages, max_ctx_len) -> int:
    mc, ac = mamba_cfg(cfg), attn_cfg(cfg, max_pages, num_pages)
    return lib().hspec_drafter_forward_workspace(C.byref(mc), C.byref(ac), cfg.d_ff, int(max_ctx_len))


def drafter_forward(cfg, shared: dict, layers: list, X: dict, out, ws, max_ctx_len: int):
    """out [B, k, d_model] fp32 = the whole drafter over the block (hspec_drafter_forward).
    ``shared``: W_r, W_dS (or W_dS_packed); ``layers``: per-layer weight dicts of device tensors
    with "cache" = index into X["caches"] (None: no attention)."""
    mc = mamba_cfg(cfg, shared)
    ac = attn_cfg(cfg, X["page_table"].shape[1], X["caches"][0]["k_cache"].shape[0])
    keep = []
    arr = (LayerW * len(layers))()
    for i, W in enumerate(layers):
        mw = mamba_w(W) if W.get("W_in") is not None else None
        keep.append(mw)
        aw = None
        c = None
        if W.get("cache") is not None:
            aw = attn_w(W)
            keep.append(aw)
            c = X["caches"][W["cache"]]
        arr[i] = LayerW(C.pointer(mw) if mw is not None else None, ptr(W.get("norm1_w")),
                        C.pointer(aw) if aw is not None else None,
                        ptr(W.get("norm2_w")) if aw is not None else None, ptr(c["k_cache"]) if c else None,
                        ptr(c["v_cache"]) if c else None, ptr(W["norm3_w"]), ptr(W["W_gate"]), ptr(W["W_up"]),
                        ptr(W["W_down"]))
    W_dS = shared.get("W_dS_packed", shared.get("W_dS"))
    if "W_r" not in shared:
        shared = dict(shared, W_r=None)
    _check(lib().hspec_drafter_forward(C.byref(mc), C.byref(ac), cfg.d_ff, len(layers), ptr(shared["W_r"]), ptr(W_dS),
                                       arr, ptr(X.get("h_last")), ptr(X["block_emb"]), ptr(X["page_table"]),
                                       ptr(X["ctx_lens"]), int(max_ctx_len), ptr(out), ptr(ws), ws.numel(),
                                       stream_ptr()))


def kv_inject_workspace(cfg, max_pages, num_pages) -> int:
    ac = attn_cfg(cfg, max_pages, num_pages)
    return lib().hspec_kv_inject_workspace(C.byref(ac), cfg.d_h)


def kv_inject(cfg, IW: dict, h_new, caches: list, page_table, ctx_lens, ws):
    """Drafter-side KV injection (hspec_kv_inject): appends cfg.k new positions per request to
    each layer's cache in ``caches`` (dicts of k_cache/v_cache device tensors, in place)."""
    n = len(IW["layers"])
    ac = attn_cfg(cfg, page_table.shape[1], caches[0]["k_cache"].shape[0])
    arr = lambda xs: (C.c_void_p * n)(*[x.data_ptr() for x in xs])  # noqa: E731
    L = IW["layers"]
    _check(lib().hspec_kv_inject(C.byref(ac), cfg.d_h, n, ptr(h_new), ptr(IW["W_fc"]), arr([w["W_k"] for w in L]),
                                 arr([w["W_v"] for w in L]), arr([w["k_norm_w"] for w in L]),
                                 arr([c["k_cache"] for c in caches]), arr([c["v_cache"] for c in caches]),
                                 ptr(page_table), ptr(ctx_lens), ptr(ws), ws.numel(), stream_ptr()))


# ----------------------------------------------------------------- the target's side of a step

def _dev() -> int:
    return _torch().cuda.current_device()


def _arg(name, t, dtype, shape, dev):
    """Address of a contiguous tensor of this type and shape on device `dev` (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on the current device, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _run(fn, dev, ws, *args):
    """One call on the current stream of `dev`, with workspace `ws` (uint8, on the same device)."""
    torch = _torch()
    if ws.dtype is not torch.uint8 or ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws: expected a contiguous uint8 tensor on the current device")
    _check(fn(*args, ws.data_ptr(), ws.numel(), torch.cuda.current_stream(dev).cuda_stream))


def _storage(dtype: int):
    torch = _torch()
    return torch.float32 if dtype == F32 else torch.bfloat16


def chunk_cfg(B, T, max_new, Hq, Hkv, D, page_size, max_pages, num_pages, dtype=BF16, window=0, eps=1e-6, scale=0.0,
              rope_theta=1e6) -> ChunkCfg:
    """A ragged batch of new tokens over a paged cache (hspec_chunk_cfg)."""
    return ChunkCfg(B, T, max_new, Hq, Hkv, D, page_size, max_pages, num_pages, window, dtype, eps, scale, rope_theta)


def chunk_append_workspace(cc: ChunkCfg) -> int:
    return lib().hspec_chunk_append_workspace(C.byref(cc))


def chunk_append(cc: ChunkCfg, qkv, cu_new, ctx_lens, q, k_cache, v_cache, page_table, ws, q_norm_w=None, k_norm_w=None):
    """Norm and RoPE of the new tokens' q and k; q out, K and V into the pages (hspec_chunk_append)."""
    torch = _torch()
    dev, i32, f32, st = _dev(), torch.int32, torch.float32, _storage(cc.dtype)
    B, T, Hq, Hkv, D = cc.B, cc.T, cc.Hq, cc.Hkv, cc.D
    pool = (cc.num_pages, cc.page_size, Hkv, D)
    code = F32 if qkv.dtype is f32 else BF16
    _run(lib().hspec_chunk_append, dev, ws, C.byref(cc), code,
         _arg("qkv", qkv, _storage(code), (T, (Hq + 2 * Hkv) * D), dev), _arg("q_norm_w", q_norm_w, f32, (D,), dev),
         _arg("k_norm_w", k_norm_w, f32, (D,), dev), _arg("cu_new", cu_new, i32, (B + 1,), dev),
         _arg("ctx_lens", ctx_lens, i32, (B,), dev), _arg("q", q, st, (T, Hq, D), dev),
         _arg("k_cache", k_cache, st, pool, dev), _arg("v_cache", v_cache, st, pool, dev),
         _arg("page_table", page_table, i32, (B, cc.max_pages), dev))


def chunk_attn_workspace(cc: ChunkCfg, max_len: int) -> int:
    return lib().hspec_chunk_attn_workspace(C.byref(cc), int(max_len))


def chunk_attn(cc: ChunkCfg, q, cu_new, k_cache, v_cache, page_table, ctx_lens, max_len: int, o, ws):
    """o [T, Hq, D] = causal attention of the new tokens over the paged cache (hspec_chunk_attn)."""
    torch = _torch()
    dev, i32, st = _dev(), torch.int32, _storage(cc.dtype)
    B, rows, pool = cc.B, (cc.T, cc.Hq, cc.D), (cc.num_pages, cc.page_size, cc.Hkv, cc.D)
    _run(lib().hspec_chunk_attn, dev, ws, C.byref(cc), _arg("q", q, st, rows, dev),
         _arg("cu_new", cu_new, i32, (B + 1,), dev), _arg("k_cache", k_cache, st, pool, dev),
         _arg("v_cache", v_cache, st, pool, dev), _arg("page_table", page_table, i32, (B, cc.max_pages), dev),
         _arg("ctx_lens", ctx_lens, i32, (B,), dev), int(max_len), _arg("o", o, st, rows, dev))


def verify_cfg(B, k, rows, vocab, draft_vocab, dtype=BF16, temperature=1.0, draft_temperature=1.0) -> VerifyCfg:
    return VerifyCfg(B, k, rows, vocab, draft_vocab, dtype, temperature, draft_temperature)


def verify_workspace(vc: VerifyCfg) -> int:
    return lib().hspec_verify_workspace(C.byref(vc))


def verify(vc: VerifyCfg, target_logits, draft_tokens, tokens, n_accepted, ws, draft_logits=None, cu_rows=None, d2t=None,
           t2d=None, u=None, gumbel=None):
    """tokens [B, k+1], n_accepted [B] = which drafts stand against the target (hspec_verify)."""
    torch = _torch()
    dev, i32, f32 = _dev(), torch.int32, torch.float32
    B, k, V, Vd = vc.B, vc.k, vc.vocab, vc.draft_vocab
    _run(lib().hspec_verify, dev, ws, C.byref(vc),
         _arg("target_logits", target_logits, _storage(vc.dtype), (vc.rows, V), dev),
         _arg("draft_logits", draft_logits, f32, (B, k, Vd), dev), _arg("draft_tokens", draft_tokens, i32, (B, k), dev),
         _arg("cu_rows", cu_rows, i32, (B + 1,), dev), _arg("d2t", d2t, i32, (Vd,), dev), _arg("t2d", t2d, i32, (V,), dev),
         _arg("u", u, f32, (B, k), dev), _arg("gumbel", gumbel, f32, (B, V), dev),
         _arg("tokens", tokens, i32, (B, k + 1), dev), _arg("n_accepted", n_accepted, i32, (B,), dev))


# ------------------------------------------------------------ the target's cache in 4 bits

def mx_cache_shape(cc: ChunkCfg) -> tuple:
    """Shape of a 4-bit cache (uint8): for each page and KV head the rows' codes, then their scales."""
    return cc.num_pages, cc.Hkv, cc.page_size * (cc.D // 2 + cc.D // 32)


def chunk_append_mx_workspace(cc: ChunkCfg) -> int:
    return lib().hspec_chunk_append_mx_workspace(C.byref(cc))


def chunk_append_mx(cc: ChunkCfg, qkv, cu_new, ctx_lens, q, k_cache, v_cache, page_table, ws, q_norm_w=None, k_norm_w=None):
    """Norm and RoPE of the new tokens' q and k; q out, K and V in 4 bits into the pages (hspec_chunk_append_mx)."""
    torch = _torch()
    dev, i32, f32, u8, st = _dev(), torch.int32, torch.float32, torch.uint8, _storage(cc.dtype)
    B, T, Hq, Hkv, D, pool = cc.B, cc.T, cc.Hq, cc.Hkv, cc.D, mx_cache_shape(cc)
    code = F32 if qkv.dtype is f32 else BF16
    _run(lib().hspec_chunk_append_mx, dev, ws, C.byref(cc), code,
         _arg("qkv", qkv, _storage(code), (T, (Hq + 2 * Hkv) * D), dev), _arg("q_norm_w", q_norm_w, f32, (D,), dev),
         _arg("k_norm_w", k_norm_w, f32, (D,), dev), _arg("cu_new", cu_new, i32, (B + 1,), dev),
         _arg("ctx_lens", ctx_lens, i32, (B,), dev), _arg("q", q, st, (T, Hq, D), dev),
         _arg("k_cache", k_cache, u8, pool, dev), _arg("v_cache", v_cache, u8, pool, dev),
         _arg("page_table", page_table, i32, (B, cc.max_pages), dev))


def chunk_read_mx_workspace(cc: ChunkCfg) -> int:
    return lib().hspec_chunk_read_mx_workspace(C.byref(cc))


def chunk_read_mx(cc: ChunkCfg, cu_new, ctx_lens, k_cache, v_cache, page_table, k, v, ws):
    """k, v [T, Hkv, D] = what the 4-bit caches hold at the rows' positions (hspec_chunk_read_mx)."""
    torch = _torch()
    dev, i32, u8, st = _dev(), torch.int32, torch.uint8, _storage(cc.dtype)
    B, pool, rows = cc.B, mx_cache_shape(cc), (cc.T, cc.Hkv, cc.D)
    _run(lib().hspec_chunk_read_mx, dev, ws, C.byref(cc), _arg("cu_new", cu_new, i32, (B + 1,), dev),
         _arg("ctx_lens", ctx_lens, i32, (B,), dev), _arg("k_cache", k_cache, u8, pool, dev),
         _arg("v_cache", v_cache, u8, pool, dev), _arg("page_table", page_table, i32, (B, cc.max_pages), dev),
         _arg("k", k, st, rows, dev), _arg("v", v, st, rows, dev))


def chunk_attn_mx_workspace(cc: ChunkCfg, max_len: int) -> int:
    return lib().hspec_chunk_attn_mx_workspace(C.byref(cc), int(max_len))


def chunk_attn_mx(cc: ChunkCfg, q, cu_new, k_cache, v_cache, page_table, ctx_lens, max_len: int, o, ws, k_new=None,
                  v_new=None, block=False):
    """o [T, Hq, D] = attention of the new tokens over the 4-bit paged cache, their own K and V in it or beside it
    (hspec_chunk_attn_mx); block: every new token of a request sees all of them."""
    torch = _torch()
    dev, i32, u8, st = _dev(), torch.int32, torch.uint8, _storage(cc.dtype)
    B, rows, new, pool = cc.B, (cc.T, cc.Hq, cc.D), (cc.T, cc.Hkv, cc.D), mx_cache_shape(cc)
    _run(lib().hspec_chunk_attn_mx, dev, ws, C.byref(cc), _arg("q", q, st, rows, dev),
         _arg("cu_new", cu_new, i32, (B + 1,), dev), _arg("k_new", k_new, st, new, dev), _arg("v_new", v_new, st, new, dev),
         CHUNK_BLOCK if block else 0, _arg("k_cache", k_cache, u8, pool, dev), _arg("v_cache", v_cache, u8, pool, dev),
         _arg("page_table", page_table, i32, (B, cc.max_pages), dev), _arg("ctx_lens", ctx_lens, i32, (B,), dev),
         int(max_len), _arg("o", o, st, rows, dev))


# ------------------------------------------------------------- logits before verification

def adjust_cfg(B, k, rows, vocab, draft_vocab=0, max_hist=0, n_bias=0, masks=0, dtype=BF16, out_dtype=BF16) -> AdjustCfg:
    return AdjustCfg(B, k, rows, vocab, draft_vocab, max_hist, n_bias, masks, dtype, out_dtype)


def adjust_logits_workspace(ac: AdjustCfg) -> int:
    return lib().hspec_adjust_logits_workspace(C.byref(ac))


def adjust_logits(ac: AdjustCfg, logits, out, ws, cu_rows=None, draft_tokens=None, d2t=None, history=None, hist_lens=None,
                  prompt_lens=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, mask=None,
                  mask_rows=None):
    """out [rows, vocab] = logits with bias, penalties and mask (hspec_adjust_logits); out may be logits."""
    torch = _torch()
    dev, i32, f32 = _dev(), torch.int32, torch.float32
    B, V = ac.B, ac.vocab
    _run(lib().hspec_adjust_logits, dev, ws, C.byref(ac), _arg("logits", logits, _storage(ac.dtype), (ac.rows, V), dev),
         _arg("cu_rows", cu_rows, i32, (B + 1,), dev), _arg("draft_tokens", draft_tokens, i32, (B, ac.k), dev),
         _arg("d2t", d2t, i32, (ac.draft_vocab,), dev), _arg("history", history, i32, (B, ac.max_hist), dev),
         _arg("hist_lens", hist_lens, i32, (B,), dev), _arg("prompt_lens", prompt_lens, i32, (B,), dev),
         _arg("repetition", repetition, f32, (B,), dev), _arg("frequency", frequency, f32, (B,), dev),
         _arg("presence", presence, f32, (B,), dev), _arg("bias_ids", bias_ids, i32, (B, ac.n_bias), dev),
         _arg("bias", bias, f32, (B, ac.n_bias), dev), _arg("mask", mask, i32, (ac.masks, (V + 31) // 32), dev),
         _arg("mask_rows", mask_rows, i32, (ac.rows,), dev), _arg("out", out, _storage(ac.out_dtype), (ac.rows, V), dev))
