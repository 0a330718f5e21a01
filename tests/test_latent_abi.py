"""CPU checks of the latent attention entry points and the norm with a residual:
exported as declared, refusals on the host (every case returns before any CUDA
call), tensors that are shorter than the call says."""
import os
import re

import pytest
import torch

import paper_2607_12875_gb300 as gb
from paper_2607_12875_gb300 import attn, latent
from test_attn_abi import Rows as Anything, Ws, changed, status_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gblatent.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gb.LIB_PATH):
        from paper_2607_12875_gb300 import build
        build.build()
    return gb.lib()


def test_header_binding_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^[A-Za-z_][\w \t\*]*?\b(latent_\w+)\s*\(", text, flags=re.M)
    assert set(names) == set(latent.LATENT_EXPORTS)
    for n in names:
        assert hasattr(lib, n)


def cfg(**kw):
    c = gb.latent_config(8)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("change,status", [
    ({}, gb.OK),
    (dict(heads=0), gb.EINVAL), (dict(heads=4097), gb.EUNSUPPORTED),
    (dict(latent_dim=0), gb.EINVAL), (dict(latent_dim=500), gb.EUNSUPPORTED), (dict(latent_dim=520), gb.EUNSUPPORTED),
    (dict(rope_dim=0), gb.OK), (dict(rope_dim=-16), gb.EINVAL), (dict(rope_dim=24), gb.EUNSUPPORTED),
    (dict(rope_dim=144), gb.EUNSUPPORTED),
    (dict(nope_dim=0), gb.EINVAL), (dict(nope_dim=132), gb.EUNSUPPORTED), (dict(nope_dim=136), gb.EUNSUPPORTED),
    (dict(value_dim=0), gb.EINVAL), (dict(value_dim=12), gb.EUNSUPPORTED), (dict(value_dim=256), gb.EUNSUPPORTED),
    (dict(act_dtype=2), gb.EINVAL), (dict(causal=2), gb.EINVAL), (dict(scale=float("inf")), gb.EINVAL),
    (dict(rotary_scale=float("nan")), gb.EINVAL), (dict(rotary_layout=2), gb.EINVAL), (dict(norm_eps=-1.0), gb.EINVAL),
    (dict(norm_eps=float("nan")), gb.EINVAL), (dict(page=0), gb.EINVAL), (dict(page=48), gb.EUNSUPPORTED),
])
def test_configs(lib, change, status):
    c = cfg(**change)
    assert gb.latent_check_config(c) == status
    assert (gb.latent_workspace_size(c, 4, 2) > 0) == (status == gb.OK)


def test_workspace_sizes(lib):
    assert gb.latent_workspace_size(cfg(), -1, 2) == 0 and gb.latent_workspace_size(cfg(), 4, -2) == 0
    assert gb.latent_workspace_size(cfg(), 0, 0) > 0


class Rows(Anything):
    """bf16 elements."""

    def element_size(self):
        return 2


class Array(Anything):
    """n entries of so many bytes at an address that is never read here."""

    def __init__(self, n, size=4, at=0x1000):
        super().__init__(n, 1, 1, at)
        self.size = size

    def element_size(self):
        return self.size

    def is_contiguous(self):
        return True


class Flat(Rows):
    def __init__(self, T=4, D=576, at=0x1000, strides=None):
        super().__init__(T, 1, D, at)
        self.shape, self.strides = (T, D), strides or (D, 1)


def batch(**kw):
    return changed(attn.AttnBatch(2, 3, 0x1000, 0x2000, 0x3000), **kw)


def pool(at=0x5000, n=10):
    return latent.LatentCache(at, n)


def test_append_refusals(lib):
    table, gamma = Array(64, 8), Array(512, 2)

    def call(c=cfg(), b=batch(), kv=Flat(), gamma=gamma, table=table, cache=pool(), **kw):
        return status_of(gb.latent_append, c, b, kv, gamma, table, cache, **kw)
    q = Rows(D=64)
    assert call(table=None) == gb.EINVAL
    assert call(table=Array(64, 8, 0x1008)) == gb.EINVAL
    assert call(gamma=Array(512, 2, 0x1004)) == gb.EINVAL
    assert call(kv=Flat(at=0x1002)) == gb.EINVAL
    assert call(kv=Flat(strides=(577, 1))) == gb.EINVAL
    assert call(kv_out=Flat(strides=(64, 1))) == gb.EINVAL             # rows that overlap
    assert call(q_out=q) == gb.EINVAL                                  # no q to turn
    assert call(q=q, q_out=Rows(D=64, strides=(64, 64, 1))) == gb.EINVAL
    assert call(q=Rows(D=64, strides=(516, 64, 1)), q_out=q) == gb.EINVAL
    assert call(positions=Array(4, at=0x1001)) == gb.EINVAL
    assert call(cache=pool(None)) == gb.EINVAL and call(cache=pool(0x5004)) == gb.EINVAL and call(cache=pool(n=-1)) == gb.EINVAL
    assert call(cache=pool(n=(1 << 24) + 1)) == gb.EUNSUPPORTED
    for kw in (dict(cu_q=None), dict(kv_len=0x1001), dict(page_table=None), dict(B=-1), dict(max_pages=-1)):
        assert call(b=batch(**kw)) == gb.EINVAL, kw
    assert call(b=batch(B=0)) == gb.OK and call(kv=Flat(T=0)) == gb.OK  # nothing to do
    c0 = cfg(rope_dim=0)
    assert gb.lib().latent_append(c0, 4, batch(), latent._flat(Flat(D=512), 4, 512), None, attn._rows(q, 4, 8, 0), None, None,
                                  pool(), None, attn._rows(q, 4, 8, 0), None) == gb.EINVAL   # nothing turns
    with pytest.raises(ValueError):
        call(q=q)                                                      # turned into what?


def test_attention_refusals(lib):
    c = cfg()
    ws = Ws(gb.latent_workspace_size(c, 4, 2))
    q, k, kr, v, out = Rows(D=192), Rows(), Flat(D=64), Rows(), Rows()

    def prompt(q=q, k=k, kr=kr, v=v, cu=Array(3), out=out, ws=ws, c=c, **kw):
        return status_of(gb.latent_prompt, c, q, k, kr, v, cu, cu, out, ws, **kw)
    assert prompt(ws=Ws(64)) == gb.EWORKSPACE and prompt(ws=Ws(1 << 40, at=0x10010)) == gb.EINVAL
    assert prompt(cu=Array(3, at=0x1002)) == gb.EINVAL
    assert prompt(q=Rows(D=192, at=0x1008)) == gb.EINVAL
    assert prompt(out=Rows(strides=(1024, 64, 1))) == gb.EINVAL
    assert prompt(k=Rows(strides=(1028, 128, 1))) == gb.EINVAL
    assert prompt(kr=Flat(D=64, at=0x1004)) == gb.EINVAL and prompt(kr=None) == gb.EINVAL
    assert prompt(v=Rows(at=0x1002)) == gb.EINVAL and prompt(lse=Array(32, at=0x1002)) == gb.EINVAL
    assert prompt(cu=Array(1)) == gb.OK and prompt(q=Rows(T=0, D=192)) == gb.OK
    assert prompt(c=cfg(page=48)) == gb.EUNSUPPORTED

    wide, low = Rows(D=576), Rows(D=512)

    def cached(b=batch(), q=wide, cache=pool(), out=low, ws=ws, c=c, **kw):
        return status_of(gb.latent_cached, c, b, q, cache, out, ws, **kw)
    assert cached(ws=Ws(64)) == gb.EWORKSPACE
    assert cached(cache=pool(0x5008)) == gb.EINVAL and cached(b=batch(kv_len=None)) == gb.EINVAL
    assert cached(out=Rows(D=512, at=0x1004)) == gb.EINVAL and cached(out=Rows(D=512, strides=(4096, 256, 1))) == gb.EINVAL
    assert cached(lse=Array(32, at=0x1001)) == gb.EINVAL
    assert cached(b=batch(B=0)) == gb.OK
    assert cached(b=batch(max_pages=(1 << 24) + 1)) == gb.EUNSUPPORTED
    assert cached(cache=pool(n=(1 << 24) + 1)) == gb.EUNSUPPORTED
    many = Rows(T=(1 << 27) + 1, D=576)
    assert cached(q=many, out=Rows(T=(1 << 27) + 1, D=512)) == gb.EUNSUPPORTED


def test_tensors_that_do_not_fit_are_refused():
    c = gb.latent_config(8, latent_dim=64, rope_dim=16, nope_dim=32, value_dim=32, page=16)
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    b = gb.attn_batch(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32))
    cu, ws, cache, table = torch.zeros(3, dtype=torch.int32), torch.zeros(64), gb.latent_cache(t(4, 16, 80)), torch.zeros(8, dtype=torch.int64)
    bad = [
        lambda: gb.latent_append(c, b, t(5, 72), t(64), table, cache),
        lambda: gb.latent_append(c, b, t(5, 80), t(60), table, cache),
        lambda: gb.latent_append(c, b, t(5, 80), t(64), table[:4], cache),
        lambda: gb.latent_append(c, b, t(5, 80), t(64), table, cache, q=t(4, 8, 16), q_out=t(5, 8, 16)),
        lambda: gb.latent_append(c, b, t(5, 80), t(64), table, cache, kv_out=t(4, 80)),
        lambda: gb.latent_append(c, b, t(5, 160)[:, ::2], t(64), table, cache),
        lambda: gb.latent_append(c, b, t(5, 80), t(64), table, gb.latent_cache(t(4, 16, 96))),
        lambda: gb.latent_append(c, b, t(5, 80), t(64), table, gb.latent_cache(t(4, 32, 80))),
        lambda: gb.latent_cache(t(4, 16, 160)[..., :80]), lambda: gb.latent_cache(t(4, 80)),
        lambda: gb.latent_prompt(c, t(5, 8, 48), t(7, 8, 32), t(6, 16), t(7, 8, 32), cu, cu, t(5, 8, 32), ws),
        lambda: gb.latent_prompt(c, t(5, 8, 48), t(7, 8, 32), t(7, 16), t(6, 8, 32), cu, cu, t(5, 8, 32), ws),
        lambda: gb.latent_prompt(c, t(5, 8, 40), t(7, 8, 32), t(7, 16), t(7, 8, 32), cu, cu, t(5, 8, 32), ws),
        lambda: gb.latent_prompt(c, t(5, 8, 48), t(7, 8, 32), t(7, 16), t(7, 8, 32), cu, cu[:2], t(5, 8, 32), ws),
        lambda: gb.latent_prompt(c, t(5, 8, 48), t(7, 8, 32), t(7, 16), t(7, 8, 32), cu, cu, t(4, 8, 32), ws),
        lambda: gb.latent_cached(c, b, t(5, 8, 64), cache, t(5, 8, 64), ws),
        lambda: gb.latent_cached(c, b, t(5, 8, 80), cache, t(5, 7, 64), ws),
        lambda: gb.latent_cached(c, b, t(5, 8, 80), cache, t(5, 8, 64), ws, lse=torch.zeros(5, 7)),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()


def test_norm_refusals(lib):
    c = gb.make_config(4, 256, 128, 8, 2)
    x, n = 0x100000, 4 * 256 * 2

    def call(x=x, r=2 * x, g=3 * x, eps=1e-6, s=4 * x, y=5 * x, codes=6 * x, scales=7 * x, c=c):
        return gb.lib().moe_rmsnorm_add(c, x, r, g, eps, s, y, codes, scales, None)
    assert call(eps=-1.0) == gb.EINVAL and call(eps=float("nan")) == gb.EINVAL
    assert call(x=None) == gb.EINVAL and call(g=None) == gb.EINVAL
    assert call(y=None, codes=None, scales=None) == gb.EINVAL      # no output
    assert call(codes=None) == gb.EINVAL and call(scales=None) == gb.EINVAL
    for kw in (dict(x=x + 8), dict(r=2 * x + 8), dict(g=3 * x + 2), dict(s=4 * x + 8), dict(y=5 * x + 4), dict(codes=6 * x + 8),
               dict(scales=7 * x + 2)):
        assert call(**kw) == gb.EINVAL, kw
    for kw in (dict(y=x), dict(y=2 * x), dict(s=x + 16), dict(s=3 * x), dict(y=4 * x + n - 16), dict(codes=5 * x + n // 2),
               dict(scales=6 * x + 512), dict(codes=x), dict(s=2 * x + n - 16)):
        assert call(**kw) == gb.EINVAL, kw
    assert call(c=gb.make_config(4, 300, 128, 8, 2)) == gb.EUNSUPPORTED
    assert call(c=gb.make_config(0, 256, 128, 8, 2)) == gb.OK
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    for kw in (dict(x=t(3, 256)), dict(residual=t(4, 128)), dict(gamma=t(128)), dict(sum_out=t(4, 512)[:, ::2]), dict(y=t(2, 256)),
               dict(codes=t(4, 200), scales=t(8)), dict(codes=t(4, 256), scales=t(7))):
        with pytest.raises(ValueError):
            gb.moe_rmsnorm_add(c, **{**dict(x=t(4, 256), residual=t(4, 256), gamma=t(256), eps=1e-6, sum_out=t(4, 256), y=t(4, 256)), **kw})
