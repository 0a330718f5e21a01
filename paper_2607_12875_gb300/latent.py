"""Binding of latent attention (C ABI in include/gblatent.h): appending latents to
a paged cache, attention over packed prompts with expanded keys and values, and
over the cached latents themselves. Argument marshalling only, as in attn:
tensors with heads are [tokens, heads, dim], without [tokens, dim] (any strides
with contiguous last elements); handles are made once with latent_config,
latent_cache and attn_batch. A tensor that has fewer tokens, heads or elements than
the call says, or elements of another size, is refused here (ValueError)."""
from __future__ import annotations

import ctypes
import math

import paper_2607_12875_gb300 as _gb

from .attn import LAYOUTS, AttnBatch, AttnRows, _rows

# every function include/gblatent.h declares
LATENT_EXPORTS = ("latent_check_config", "latent_workspace_size", "latent_append", "latent_prompt", "latent_cached")

_i32, _vp = ctypes.c_int32, ctypes.c_void_p


class LatentConfig(ctypes.Structure):
    _fields_ = [("heads", _i32), ("latent_dim", _i32), ("rope_dim", _i32), ("nope_dim", _i32), ("value_dim", _i32),
                ("act_dtype", _i32), ("causal", _i32), ("scale", ctypes.c_float), ("rotary_layout", _i32),
                ("rotary_scale", ctypes.c_float), ("norm_eps", ctypes.c_float), ("page", _i32)]


class LatentCache(ctypes.Structure):
    _fields_ = [("rows", _vp), ("n_pages", _i32)]


def _bind(L) -> None:
    """Argument types of the latent attention entry points of the loaded library."""
    cfgp, rp, bp = ctypes.POINTER(LatentConfig), ctypes.POINTER(AttnRows), ctypes.POINTER(AttnBatch)
    cp, sz = ctypes.POINTER(LatentCache), ctypes.c_size_t
    L.latent_check_config.argtypes = [cfgp]
    L.latent_workspace_size.argtypes = [cfgp, _i32, _i32]
    L.latent_workspace_size.restype = sz
    L.latent_append.argtypes = [cfgp, _i32, bp, rp, _vp, rp, _vp, _vp, cp, rp, rp, _vp]
    L.latent_prompt.argtypes = [cfgp, _i32, _i32, _i32, rp, rp, rp, rp, _vp, _vp, rp, _vp, _vp, sz, _vp]
    L.latent_cached.argtypes = [cfgp, _i32, bp, rp, cp, rp, _vp, _vp, sz, _vp]


def latent_config(heads, *, latent_dim=512, rope_dim=64, nope_dim=128, value_dim=128, act="bf16", causal=True, scale=None,
                  rotary_layout="interleaved", rotary_scale=1.0, norm_eps=1e-6, page=64) -> LatentConfig:
    """scale None: 1/sqrt(nope_dim + rope_dim), in both forms."""
    return LatentConfig(heads, latent_dim, rope_dim, nope_dim, value_dim, _gb.DTYPES[act], int(bool(causal)),
                        1.0 / math.sqrt(nope_dim + rope_dim) if scale is None else scale, LAYOUTS[rotary_layout], rotary_scale,
                        norm_eps, page)


def latent_check_config(cfg: LatentConfig) -> int:
    return _gb.lib().latent_check_config(ctypes.byref(cfg))


def latent_workspace_size(cfg: LatentConfig, T: int, B: int) -> int:
    return _gb.lib().latent_workspace_size(ctypes.byref(cfg), T, B)


def latent_cache(pool) -> LatentCache:
    """Pointer bundle of a pool of cache pages [n_pages, page, latent_dim + rope_dim] (the tensor must stay alive)."""
    if len(pool.shape) != 3 or not pool.is_contiguous():
        raise ValueError("a pool of pages is contiguous, [n_pages, page, latent_dim + rope_dim]")
    c = LatentCache(_gb._ptr(pool), pool.shape[0])
    c.shape = (*pool.shape[1:], pool.element_size())  # (the calls hold it against their config)
    return c


def _pool(page, width, size, cache):
    want = (page, width, size)
    if getattr(cache, "shape", want) != want:
        raise ValueError(f"pages of {cache.shape} (tokens, elements, bytes of one) in a call of {want}")
    return cache


def _sized(size, *tensors):
    for t in tensors:
        if t is not None and t.element_size() != size:
            raise ValueError(f"elements of {t.element_size()} bytes in a call of {size}")


def _vector(t, n, size):
    """Address of an array of at least n entries of so many bytes (None: no array)."""
    if t is None:
        return None
    if t.numel() < n or t.element_size() != size or not t.is_contiguous():
        raise ValueError(f"{t.numel()} entries of {t.element_size()} bytes, or not contiguous, where the call takes {n} of {size}")
    return t.data_ptr()


def _flat(t, tokens, dim):
    """Rows without heads."""
    if t is None:
        return None
    n, d = t.shape
    if n < tokens or d < dim:
        raise ValueError(f"[{n}, {d}] rows in a call of {tokens} tokens of {dim}")
    ts, one = t.stride()
    if one != 1:
        raise ValueError("the elements of a row are not contiguous")
    r = AttnRows()
    r.data, r.token_stride = t.data_ptr(), ts
    return r


def latent_append(cfg, batch, kv, gamma, table, cache, q=None, q_out=None, kv_out=None, positions=None, stream=None):
    """gamma None: the latent is stored as it is; q_out and kv_out are optional."""
    T, R, H, P, size = kv.shape[0], cfg.latent_dim, cfg.heads, cfg.rope_dim, 4 if cfg.act_dtype == _gb.F32 else 2
    W = R + P
    if q is not None and q_out is None:
        raise ValueError("queries are turned into q_out")
    _sized(size, kv, q, q_out, kv_out)
    _gb._check(_gb.lib().latent_append(cfg, T, batch, _flat(kv, T, W), _vector(gamma, R, size),
                                       _rows(q, T, H, P), _vector(positions, T, 4), _vector(table, P // 2, 8), _pool(cfg.page, W, size, cache),
                                       _flat(kv_out, T, W), _rows(q_out, T, H, P), _gb._stream(stream)), "latent_append")


def latent_prompt(cfg, q, k, k_rope, v, cu_q, cu_k, out, ws, lse=None, stream=None):
    """k_rope may be None where the config has no rotary elements."""
    Tq, Tk, B, H, N = q.shape[0], k.shape[0], cu_q.numel() - 1, cfg.heads, cfg.nope_dim
    _sized(4 if cfg.act_dtype == _gb.F32 else 2, q, k, k_rope, v, out)
    _gb._check(_gb.lib().latent_prompt(cfg, Tq, Tk, B, _rows(q, Tq, H, N + cfg.rope_dim), _rows(k, Tk, H, N),
                                       _flat(k_rope, Tk, cfg.rope_dim), _rows(v, Tk, H, cfg.value_dim), _vector(cu_q, B + 1, 4),
                                       _vector(cu_k, B + 1, 4), _rows(out, Tq, H, cfg.value_dim), _vector(lse, Tq * H, 4), _gb._ptr(ws),
                                       ws.numel() * ws.element_size(), _gb._stream(stream)), "latent_prompt")


def latent_cached(cfg, batch, q, cache, out, ws, lse=None, stream=None):
    T, H, R, size = q.shape[0], cfg.heads, cfg.latent_dim, 4 if cfg.act_dtype == _gb.F32 else 2
    W = R + cfg.rope_dim
    _sized(size, q, out)
    _gb._check(_gb.lib().latent_cached(cfg, T, batch, _rows(q, T, H, W), _pool(cfg.page, W, size, cache),
                                       _rows(out, T, H, R), _vector(lse, T * H, 4), _gb._ptr(ws),
                                       ws.numel() * ws.element_size(), _gb._stream(stream)), "latent_cached")
