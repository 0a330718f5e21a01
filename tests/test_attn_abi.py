"""CPU checks of the attention entry points: exported as declared, refusals on
the host (every case returns before any CUDA call)."""
import ctypes
import os
import re

import pytest

import paper_2607_12875_gb300 as gb
from paper_2607_12875_gb300 import attn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gbattn.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2607_12875_gb300 import build
        build.build()
    return gb.lib()


def test_header_binding_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^[A-Za-z_][\w \t\*]*?\b(attn_\w+)\s*\(", text, flags=re.M)
    assert set(names) == set(attn.ATTN_EXPORTS)
    for n in names:
        assert hasattr(lib, n)


def cfg(**kw):
    c = gb.attn_config(8, 2, 128, rotary_dim=64, cache="e4m3")
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("change,status", [
    ({}, gb.OK),
    (dict(heads_q=7), gb.EINVAL),
    (dict(heads_kv=0), gb.EINVAL),
    (dict(head_dim=0), gb.EINVAL),
    (dict(head_dim=100, rotary_dim=0), gb.EUNSUPPORTED),
    (dict(head_dim=264), gb.EUNSUPPORTED),
    (dict(heads_q=8192), gb.EUNSUPPORTED),
    (dict(act_dtype=2), gb.EINVAL),
    (dict(causal=2), gb.EINVAL),
    (dict(window=-1), gb.EINVAL),
    (dict(scale=float("nan")), gb.EINVAL),
    (dict(rotary_scale=float("inf")), gb.EINVAL),
    (dict(rotary_dim=-16), gb.EINVAL),
    (dict(rotary_dim=144), gb.EINVAL),
    (dict(rotary_dim=24), gb.EUNSUPPORTED),
    (dict(rotary_layout=2), gb.EINVAL),
    (dict(cache_dtype=2), gb.EINVAL),
    (dict(page=0), gb.EINVAL),
    (dict(page=48), gb.EUNSUPPORTED),
    (dict(page=256), gb.EUNSUPPORTED),
])
def test_configs(lib, change, status):
    c = cfg(**change)
    assert gb.attn_check_config(c) == status
    assert (gb.attn_workspace_size(c, 4, 2) > 0) == (status == gb.OK)


def test_workspace_sizes(lib):
    assert gb.attn_workspace_size(cfg(), -1, 2) == 0
    assert gb.attn_workspace_size(cfg(), 4, -2) == 0
    assert gb.attn_workspace_size(cfg(), 0, 0) > 0


class Rows:
    """Stands for a [T, H, D] tensor at an address that is never read here."""

    def __init__(self, T=4, H=8, D=128, at=0x1000, strides=None):
        self.shape, self.at, self.strides = (T, H, D), at, strides or (H * D, D, 1)

    def data_ptr(self):
        return self.at

    def stride(self):
        return self.strides

    def numel(self):
        return self.shape[0]

    def element_size(self):
        return 1


class Ws(Rows):
    def __init__(self, n, at=0x10000):
        super().__init__(at=at)
        self.n = n

    def numel(self):
        return self.n


def status_of(call, *a, **kw):
    try:
        call(*a, stream=0, **kw)
    except gb.GbmoeError as e:
        return e.status
    return gb.OK


def test_rope_refusals(lib):
    c = cfg()
    q, k, pos, tab = Rows(), Rows(H=2), Rows(), Rows()
    bad = Rows(at=0x1008)                                   # not on 16 bytes
    odd = Rows(strides=(8 * 128 + 4, 128, 1))                # rows not on 16 bytes
    over = Rows(strides=(512, 128, 1))                       # output rows that overlap
    for args in [(None, None, pos, tab, None, None), (q, None, None, tab, q, None), (q, None, pos, None, q, None),
                 (q, k, pos, tab, q, None), (bad, None, pos, tab, q, None), (q, None, pos, tab, bad, None),
                 (odd, None, pos, tab, q, None), (q, None, pos, tab, over, None),
                 (q, None, Rows(at=0x1002), tab, q, None), (q, None, pos, Rows(at=0x1004), q, None)]:
        if args[0] is None:
            st = gb.lib().attn_rope(c, 4, None, None, 0x1000, 0x1000, 0, None, None, None)
        else:
            st = status_of(gb.attn_rope, c, *args)
        assert st == gb.EINVAL, args
    assert gb.lib().attn_rope(c, 4, attn._rows(q), None, 0x1000, 0x1000, 2, attn._rows(q), None, None) == gb.EINVAL
    assert gb.lib().attn_rope(c, -1, attn._rows(q), None, 0x1000, 0x1000, 0, attn._rows(q), None, None) == gb.EINVAL
    assert gb.lib().attn_rope(c, 0, attn._rows(q), None, None, None, 0, attn._rows(q), None, None) == gb.OK


def test_rope_table_refusals(lib):
    for a in [(0, 1e4, "plain"), (7, 1e4, "plain"), (64, 1.0, "plain"), (64, float("inf"), "plain"),
              (2, 1e4, "ntk")]:
        with pytest.raises(gb.GbmoeError):
            gb.attn_rope_table(a[0], a[1], scaling=a[2], device="cpu")
    for kw in [dict(factor=0.0), dict(factor=float("nan")), dict(original_ctx=0), dict(slow=0.0), dict(slow=9.0, fast=3.0)]:
        with pytest.raises(gb.GbmoeError):
            gb.attn_rope_table(64, scaling="ramp", device="cpu", **kw)
    assert gb.lib().attn_rope_table(64, 1e4, 4, 1.0, 1.0, 1.0, 2.0, 0x1000) == gb.EINVAL
    assert gb.lib().attn_rope_table(64, 1e4, 0, 1.0, 1.0, 1.0, 2.0, None) == gb.EINVAL


def bundles():
    cache = attn.AttnCache(0x1000, 0x2000, 0x3000, 0x4000, 10)
    batch = attn.AttnBatch(2, 3, 0x1000, 0x2000, 0x3000)
    return cache, batch


def changed(struct, **kw):
    c = type(struct)()
    ctypes.pointer(c)[0] = struct
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_append_refusals(lib):
    c = cfg()
    cache, batch = bundles()
    k, v, q, tab = Rows(H=2), Rows(H=2), Rows(), Rows()

    def call(c=c, batch=batch, k=k, v=v, tab=tab, cache=cache, **kw):
        return status_of(gb.attn_append, c, batch, k, v, tab, cache, **kw)
    assert call(tab=None) == gb.EINVAL
    assert call(v=Rows(H=2, at=0x1004)) == gb.EINVAL
    assert call(q_out=q) == gb.EINVAL                        # no q to turn
    assert call(q=q, q_out=Rows(strides=(128, 128, 1))) == gb.EINVAL
    assert call(k_out=Rows(H=2, at=0x1002)) == gb.EINVAL
    assert call(positions=Rows(at=0x1001)) == gb.EINVAL
    for kw in (dict(k=None), dict(v=0x1001), dict(k_scale=None), dict(n_pages=-1)):
        assert call(cache=changed(cache, **kw)) == gb.EINVAL, kw
    for kw in (dict(cu_q=None), dict(kv_len=0x1001), dict(page_table=None), dict(B=-1), dict(max_pages=-1)):
        assert call(batch=changed(batch, **kw)) == gb.EINVAL, kw
    assert call(batch=changed(batch, B=0)) == gb.OK          # nothing to do
    assert call(k=Rows(T=0, H=2), v=Rows(T=0, H=2)) == gb.OK
    assert call(c=cfg(page=48)) == gb.EUNSUPPORTED


def test_attention_refusals(lib):
    c = cfg()
    cache, batch = bundles()
    q, k, out = Rows(), Rows(H=2), Rows()
    ws = Ws(gb.attn_workspace_size(c, 4, 2))

    def prompt(q=q, k=k, v=k, cu=Rows(T=3), out=out, ws=ws, **kw):
        return status_of(gb.attn_prompt, c, q, k, v, cu, cu, out, ws, **kw)
    assert prompt(ws=Ws(64)) == gb.EWORKSPACE
    assert prompt(ws=Ws(1 << 40, at=0x10010)) == gb.EINVAL
    assert prompt(cu=Rows(T=3, at=0x1002)) == gb.EINVAL
    assert prompt(q=Rows(at=0x1008)) == gb.EINVAL
    assert prompt(out=Rows(strides=(1024, 64, 1))) == gb.EINVAL
    assert prompt(k=Rows(H=2, strides=(260, 128, 1))) == gb.EINVAL
    assert prompt(lse=Rows(at=0x1002)) == gb.EINVAL
    assert prompt(cu=Rows(T=1)) == gb.OK                     # no sequences
    assert prompt(q=Rows(T=0)) == gb.OK

    def cached(batch=batch, q=q, cache=cache, out=out, ws=ws, **kw):
        return status_of(gb.attn_cached, c, batch, q, cache, out, ws, **kw)
    assert cached(ws=Ws(64)) == gb.EWORKSPACE
    assert cached(cache=changed(cache, v_scale=None)) == gb.EINVAL
    assert cached(batch=changed(batch, kv_len=None)) == gb.EINVAL
    assert cached(out=Rows(at=0x1004)) == gb.EINVAL
    assert cached(lse=Rows(at=0x1001)) == gb.EINVAL
    assert cached(batch=changed(batch, B=0)) == gb.OK
    with pytest.raises(ValueError):
        gb.attn_cached(c, batch, Rows(strides=(2048, 256, 2)), cache, out, ws, stream=0)


def test_sizes_that_do_not_fit_32_bits_are_refused(lib):
    c = cfg(heads_q=64, heads_kv=1, page=128)
    cache, batch = bundles()
    ws = Ws(gb.attn_workspace_size(c, 4, 2))

    def cached(T, max_pages):
        q = Rows(T=T, H=64)
        return status_of(gb.attn_cached, c, changed(batch, max_pages=max_pages), q, cache, q, ws)
    assert cached((1 << 24) + 1, 3) == gb.EUNSUPPORTED       # rows: tokens times heads of a group
    assert cached(4, (1 << 23) + 1) == gb.EUNSUPPORTED       # keys of a sequence
