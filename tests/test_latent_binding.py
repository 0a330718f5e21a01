"""CPU checks of the latent attention binding: tensors whose elements have another size than the config's, or that are
not contiguous where the call takes an array, are refused before their addresses go anywhere."""
import pytest
import torch

import paper_2607_12875_gb300 as gb


class Taken(Exception):
    """The library was called."""


class NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            raise Taken(name)
        return call


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(gb, "lib", NoLibrary)
    monkeypatch.setattr(gb, "_stream", lambda s: 0)


BF, F = torch.bfloat16, torch.float32
OTHER = {BF: F, F: BF}


def zeros(dt, *shape):
    return torch.zeros(shape, dtype=dt)


def i32(*shape):
    return zeros(torch.int32, *shape)


def config(dt):
    return gb.latent_config(8, latent_dim=64, rope_dim=16, nope_dim=32, value_dim=32, page=16, act="bf16" if dt is BF else "f32")


def append(dt, **kw):
    t = {**dict(kv=zeros(dt, 5, 80), gamma=zeros(dt, 64), table=zeros(torch.int64, 8), pool=zeros(dt, 4, 16, 80), q=zeros(dt, 5, 8, 16),
                q_out=zeros(dt, 5, 8, 16), kv_out=zeros(dt, 5, 80), positions=i32(5)), **kw}
    pool = t.pop("pool")
    gb.latent_append(config(dt), gb.attn_batch(i32(3), i32(2), i32(2, 2)), t.pop("kv"), t.pop("gamma"), t.pop("table"), gb.latent_cache(pool), **t)


def prompt(dt, **kw):
    t = {**dict(q=zeros(dt, 5, 8, 48), k=zeros(dt, 7, 8, 32), k_rope=zeros(dt, 7, 16), v=zeros(dt, 7, 8, 32), cu_q=i32(3), cu_k=i32(3),
                out=zeros(dt, 5, 8, 32), ws=zeros(F, 64), lse=zeros(F, 5, 8)), **kw}
    gb.latent_prompt(config(dt), **t)


def cached(dt, **kw):
    t = {**dict(q=zeros(dt, 5, 8, 80), pool=zeros(dt, 4, 16, 80), out=zeros(dt, 5, 8, 64), lse=zeros(F, 5, 8)), **kw}
    gb.latent_cached(config(dt), gb.attn_batch(i32(3), i32(2), i32(2, 2)), t["q"], gb.latent_cache(t["pool"]), t["out"], zeros(F, 64), lse=t["lse"])


SHAPES = [(append, "kv", (5, 80)), (append, "gamma", (64,)), (append, "pool", (4, 16, 80)), (append, "q", (5, 8, 16)),
          (append, "q_out", (5, 8, 16)), (append, "kv_out", (5, 80)), (prompt, "q", (5, 8, 48)), (prompt, "k", (7, 8, 32)),
          (prompt, "k_rope", (7, 16)), (prompt, "v", (7, 8, 32)), (prompt, "out", (5, 8, 32)), (cached, "q", (5, 8, 80)),
          (cached, "pool", (4, 16, 80)), (cached, "out", (5, 8, 64))]


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("call,name,shape", SHAPES)
def test_elements_of_another_size_are_refused(dt, call, name, shape):
    with pytest.raises(Taken):
        call(dt)
    with pytest.raises(ValueError):
        call(dt, **{name: zeros(OTHER[dt], *shape)})


@pytest.mark.parametrize("call,name,bad", [
    (append, "positions", zeros(torch.int64, 5)), (append, "positions", i32(10)[::2]), (append, "table", i32(8)),
    (append, "gamma", zeros(BF, 128)[::2]), (prompt, "cu_q", zeros(torch.int64, 3)), (prompt, "cu_k", i32(6)[::2]),
    (prompt, "lse", zeros(BF, 5, 8)), (prompt, "lse", zeros(F, 8, 5).T), (cached, "lse", zeros(torch.float64, 5, 8)),
])
def test_arrays_of_another_kind_are_refused(call, name, bad):
    with pytest.raises(ValueError):
        call(BF, **{name: bad})


def test_optional_tensors_may_be_left_out():
    with pytest.raises(Taken):
        append(BF, gamma=None, q=None, q_out=None, kv_out=None, positions=None)
    with pytest.raises(Taken):
        prompt(F, lse=None)
    with pytest.raises(Taken):
        cached(F, lse=None)


@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("name,size", [("x", 1024), ("residual", 1024), ("gamma", 256), ("sum_out", 1024), ("y", 1024)])
def test_norm_of_elements_of_another_size_is_refused(dt, name, size):
    cfg = gb.make_config(4, 256, 128, 8, 2, act="bf16" if dt is BF else "f32", w="bf16" if dt is BF else "f32")

    def call(**kw):
        t = {**dict(x=zeros(dt, 1024), residual=zeros(dt, 1024), gamma=zeros(dt, 256), eps=1e-6, sum_out=zeros(dt, 1024), y=zeros(dt, 1024),
                    codes=zeros(torch.uint8, 1024), scales=zeros(F, 8)), **kw}
        gb.moe_rmsnorm_add(cfg, **t)
    with pytest.raises(Taken):
        call()
    with pytest.raises(ValueError):
        call(**{name: zeros(OTHER[dt], size)})
    with pytest.raises(ValueError):
        call(scales=zeros(torch.float64, 8))
    with pytest.raises(ValueError):
        call(codes=zeros(torch.int32, 1024))


@pytest.mark.parametrize("dt,same", [(BF, zeros(F, 512)), (BF, zeros(torch.uint8, 4, 512)), (F, zeros(BF, 2048)), (F, zeros(torch.float64, 512))])
@pytest.mark.parametrize("name", ["x", "residual", "sum_out", "y"])
def test_norm_of_as_many_bytes_of_another_type_is_refused(dt, same, name):
    """4 rows of 256: the bytes are right, the elements are not."""
    cfg = gb.make_config(4, 256, 128, 8, 2, act="bf16" if dt is BF else "f32", w="bf16" if dt is BF else "f32")
    t = {**dict(x=zeros(dt, 1024), residual=zeros(dt, 1024), gamma=zeros(dt, 256), eps=1e-6, sum_out=zeros(dt, 1024), y=zeros(dt, 1024)), name: same}
    assert same.nbytes == 1024 * zeros(dt, 1).element_size()
    with pytest.raises(ValueError):
        gb.moe_rmsnorm_add(cfg, **t)
