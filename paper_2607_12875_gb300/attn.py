"""Binding of the attention operators (C ABI in include/gbattn.h): rotary
positions, appending to a paged cache, attention over packed prompts and over
the cache. Argument marshalling only, as in the package: q, k, v and out are
torch tensors [tokens, heads, head_dim] (any strides with contiguous heads),
handles are made once with attn_config, attn_cache and attn_batch. The library
is told one number of tokens and of heads for all tensors of a call, so a tensor
that has fewer is refused here (ValueError)."""
from __future__ import annotations

import ctypes
import math

import paper_2607_12875_gb300 as _gb

HALF, INTERLEAVED = 0, 1
CACHE_ACT, CACHE_E4M3 = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_RAMP = range(4)
LAYOUTS = {"half": HALF, "interleaved": INTERLEAVED}
CACHES = {"act": CACHE_ACT, "e4m3": CACHE_E4M3}
SCALINGS = {"plain": ROPE_PLAIN, "linear": ROPE_LINEAR, "ntk": ROPE_NTK, "ramp": ROPE_RAMP}

# every function include/gbattn.h declares
ATTN_EXPORTS = ("attn_check_config", "attn_workspace_size", "attn_rope_table", "attn_rope", "attn_append", "attn_prompt",
                "attn_cached")

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class AttnConfig(ctypes.Structure):
    _fields_ = [("heads_q", _i32), ("heads_kv", _i32), ("head_dim", _i32), ("act_dtype", _i32), ("causal", _i32),
                ("window", _i32), ("scale", ctypes.c_float), ("rotary_dim", _i32), ("rotary_layout", _i32),
                ("rotary_scale", ctypes.c_float), ("cache_dtype", _i32), ("page", _i32)]


class AttnRows(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class AttnCache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("n_pages", _i32)]


class AttnBatch(ctypes.Structure):
    _fields_ = [("B", _i32), ("max_pages", _i32), ("cu_q", _vp), ("kv_len", _vp), ("page_table", _vp)]


def _bind(L) -> None:
    """Argument types of the attention entry points of the loaded library."""
    cfgp, rp = ctypes.POINTER(AttnConfig), ctypes.POINTER(AttnRows)
    cp, bp = ctypes.POINTER(AttnCache), ctypes.POINTER(AttnBatch)
    d, sz = ctypes.c_double, ctypes.c_size_t
    L.attn_check_config.argtypes = [cfgp]
    L.attn_workspace_size.argtypes = [cfgp, _i32, _i32]
    L.attn_workspace_size.restype = sz
    L.attn_rope_table.argtypes = [_i32, d, _i32, d, d, d, d, _vp]
    L.attn_rope.argtypes = [cfgp, _i32, rp, rp, _vp, _vp, _i32, rp, rp, _vp]
    L.attn_append.argtypes = [cfgp, _i32, bp, rp, rp, rp, _vp, _vp, cp, rp, rp, _vp]
    L.attn_prompt.argtypes = [cfgp, _i32, _i32, _i32, rp, rp, rp, _vp, _vp, rp, _vp, _vp, sz, _vp]
    L.attn_cached.argtypes = [cfgp, _i32, bp, rp, cp, rp, _vp, _vp, sz, _vp]


def attn_config(heads_q, heads_kv, head_dim, *, act="bf16", causal=True, window=0, scale=None, rotary_dim=0,
                rotary_layout="half", rotary_scale=1.0, cache="act", page=64) -> AttnConfig:
    """scale None: 1/sqrt(head_dim)."""
    return AttnConfig(heads_q, heads_kv, head_dim, _gb.DTYPES[act], int(bool(causal)), window,
                      1.0 / math.sqrt(head_dim) if scale is None else scale, rotary_dim, LAYOUTS[rotary_layout], rotary_scale,
                      CACHES[cache], page)


def attn_check_config(cfg: AttnConfig) -> int:
    return _gb.lib().attn_check_config(ctypes.byref(cfg))


def attn_workspace_size(cfg: AttnConfig, T: int, B: int) -> int:
    return _gb.lib().attn_workspace_size(ctypes.byref(cfg), T, B)


def attn_rope_table(rotary_dim, base=10000.0, scaling="plain", factor=1.0, original_ctx=8192, slow=1.0, fast=32.0,
                    device="cuda"):
    """The table that attn_rope and attn_append take, as an int64 tensor [rotary_dim / 2] on the device."""
    import torch
    t = torch.empty(max(rotary_dim // 2, 1), dtype=torch.int64)
    _gb._check(_gb.lib().attn_rope_table(rotary_dim, base, SCALINGS[scaling], factor, original_ctx, slow, fast, t.data_ptr()),
               "attn_rope_table")
    return t.to(device)


def attn_cache(k, v, k_scale=None, v_scale=None) -> AttnCache:
    """Pointer bundle of a pool of cache pages [n_pages, heads_kv, page, head_dim] (tensors must stay alive)."""
    for t in (k, v):
        if t.numel() < k.numel() or not t.is_contiguous():
            raise ValueError("the pools of keys and values are contiguous and of one size")
    for t in (k_scale, v_scale):
        if t is not None and (t.numel() < math.prod(k.shape[:2]) or not t.is_contiguous()):
            raise ValueError("scales are contiguous, one for each page and kv head")
    return AttnCache(_gb._ptr(k), _gb._ptr(v), _gb._ptr(k_scale), _gb._ptr(v_scale), k.shape[0])


def attn_batch(cu_q, kv_len, page_table) -> AttnBatch:
    """Pointer bundle of a batch over the cache (int32 tensors [B + 1], [B], [B, max_pages]; they must stay alive)."""
    B = kv_len.numel()
    if cu_q.numel() < B + 1 or page_table.shape[0] < B:
        raise ValueError("a batch of B sequences has B + 1 offsets, B lengths and B rows of pages")
    for t in (cu_q, kv_len, page_table):
        if t.element_size() != 4 or not t.is_contiguous():
            raise ValueError("offsets, lengths and pages are contiguous int32 tensors")
    return AttnBatch(kv_len.numel(), page_table.shape[1], _gb._ptr(cu_q), _gb._ptr(kv_len), _gb._ptr(page_table))


def _rows(t, tokens=0, heads=0, dim=0):
    if t is None:
        return None
    if t.shape != (tokens, heads, dim):  # (more of each is fine: parts are taken)
        n, h, d = t.shape
        if n < tokens or h < heads or d < dim:
            raise ValueError(f"[{n}, {h}, {d}] rows in a call of {tokens} tokens, {heads} heads of {dim}")
    ts, hs, one = t.stride()
    if one != 1:
        raise ValueError("the elements of a head are not contiguous")
    r = AttnRows()  # (fields set one by one: 0.05 us less than through the constructor)
    r.data, r.token_stride, r.head_stride = t.data_ptr(), ts, hs
    return r


def _words(t, n):
    """Address of an array of at least n entries (None: no array)."""
    if t is not None and math.prod(t.shape) < n:
        raise ValueError(f"{math.prod(t.shape)} entries where the call takes {n}")
    return _gb._ptr(t)


def attn_rope(cfg, q, k, positions, table, q_out, k_out, inverse=False, stream=None):
    """q or k may be None (with its output)."""
    T, D = (q if q is not None else k).shape[0], cfg.head_dim
    hq, hk = cfg.heads_q, cfg.heads_kv
    _gb._check(_gb.lib().attn_rope(cfg, T, _rows(q, T, hq, D), _rows(k, T, hk, D), _words(positions, T), _gb._ptr(table),
                                   1 if inverse else 0, _rows(q_out, T, hq, D), _rows(k_out, T, hk, D),
                                   _gb._stream(stream)), "attn_rope")


def attn_append(cfg, batch, k, v, table, cache, q=None, q_out=None, k_out=None, positions=None, stream=None):
    T, hq, hk, D = k.shape[0], cfg.heads_q, cfg.heads_kv, cfg.head_dim
    _gb._check(_gb.lib().attn_append(cfg, T, batch, _rows(q, T, hq, D), _rows(k, T, hk, D), _rows(v, T, hk, D),
                                     _words(positions, T), _gb._ptr(table), cache, _rows(q_out, T, hq, D),
                                     _rows(k_out, T, hk, D), _gb._stream(stream)), "attn_append")


def attn_prompt(cfg, q, k, v, cu_q, cu_k, out, ws, lse=None, stream=None):
    Tq, Tk, B, hq, hk, D = q.shape[0], k.shape[0], cu_q.numel() - 1, cfg.heads_q, cfg.heads_kv, cfg.head_dim
    _gb._check(_gb.lib().attn_prompt(cfg, Tq, Tk, B, _rows(q, Tq, hq, D), _rows(k, Tk, hk, D), _rows(v, Tk, hk, D),
                                     _gb._ptr(cu_q), _words(cu_k, B + 1), _rows(out, Tq, hq, D), _words(lse, Tq * hq),
                                     _gb._ptr(ws), ws.numel() * ws.element_size(), _gb._stream(stream)), "attn_prompt")


def attn_cached(cfg, batch, q, cache, out, ws, lse=None, stream=None):
    T, hq, D = q.shape[0], cfg.heads_q, cfg.head_dim
    _gb._check(_gb.lib().attn_cached(cfg, T, batch, _rows(q, T, hq, D), cache, _rows(out, T, hq, D), _words(lse, T * hq),
                                     _gb._ptr(ws), ws.numel() * ws.element_size(), _gb._stream(stream)), "attn_cached")
