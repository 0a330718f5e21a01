"""CPU checks of the attention binding: tensors that are shorter than the call
says, or laid out otherwise, are refused before their addresses go anywhere."""
import pytest
import torch

import paper_2607_12875_gb300 as gb
from paper_2607_12875_gb300 import attn


class Taken(Exception):
    """The library was called."""


class NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            raise Taken(name)
        return call


STREAM = gb._stream


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(gb, "lib", NoLibrary)
    monkeypatch.setattr(gb, "_stream", lambda s: 0)


def rows(T, H, D=64):
    return torch.zeros((T, H, D), dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


CFG = gb.attn_config(8, 2, 64, rotary_dim=64, cache="e4m3", page=16)
POOL = torch.zeros((5, 2, 16, 64), dtype=torch.uint8)
SCALE = torch.zeros((5, 2), dtype=torch.uint8)
WS = torch.zeros(4096, dtype=torch.uint8)
TABLE = torch.zeros(32, dtype=torch.int64)


def batch():
    return gb.attn_batch(i32(4), i32(3), i32(3, 2))


def cache():
    return gb.attn_cache(POOL, POOL.clone(), SCALE, SCALE.clone())


def rope(q=rows(5, 8), k=rows(5, 2), pos=i32(5), q_out=rows(5, 8), k_out=rows(5, 2)):
    gb.attn_rope(CFG, q, k, pos, TABLE, q_out, k_out)


def append(k=rows(5, 2), v=rows(5, 2), q=rows(5, 8), q_out=rows(5, 8), k_out=rows(5, 2), pos=i32(5)):
    gb.attn_append(CFG, batch(), k, v, TABLE, cache(), q=q, q_out=q_out, k_out=k_out, positions=pos)


def prompt(q=rows(5, 8), k=rows(7, 2), v=rows(7, 2), cu_q=i32(4), cu_k=i32(4), out=rows(5, 8), lse=torch.zeros(5, 8)):
    gb.attn_prompt(CFG, q, k, v, cu_q, cu_k, out, WS, lse=lse)


def cached(q=rows(5, 8), out=rows(5, 8), lse=torch.zeros(5, 8)):
    gb.attn_cached(CFG, batch(), q, cache(), out, WS, lse=lse)


@pytest.mark.parametrize("call,short", [
    (rope, dict(q=rows(5, 7), q_out=rows(5, 7))), (rope, dict(q=rows(5, 8, 56))), (rope, dict(k=rows(4, 2))), (rope, dict(k=rows(5, 1))),
    (rope, dict(pos=i32(4))), (rope, dict(q_out=rows(4, 8))), (rope, dict(k_out=rows(5, 2, 32))),
    (append, dict(v=rows(4, 2))), (append, dict(v=rows(5, 1))), (append, dict(k=rows(5, 1))), (append, dict(q=rows(3, 8))),
    (append, dict(q=rows(5, 6))), (append, dict(q_out=rows(1, 8))), (append, dict(k_out=rows(4, 2))), (append, dict(pos=i32(3))),
    (prompt, dict(v=rows(6, 2))), (prompt, dict(k=rows(7, 1))), (prompt, dict(q=rows(5, 4))), (prompt, dict(out=rows(4, 8))),
    (prompt, dict(cu_k=i32(3))), (prompt, dict(lse=torch.zeros(5, 2))),
    (cached, dict(out=rows(4, 8))), (cached, dict(q=rows(5, 2))), (cached, dict(lse=torch.zeros(4, 8))),
])
def test_tensors_shorter_than_the_call_are_refused(call, short):
    with pytest.raises(Taken):
        call()
    with pytest.raises(ValueError):
        call(**short)


def test_longer_tensors_and_parts_of_wider_ones_are_taken():
    with pytest.raises(Taken):
        rope(q=rows(9, 12, 128), q_out=rows(9, 8), k=None, k_out=None, pos=i32(9))
    qkv = rows(5, 12)
    with pytest.raises(Taken):
        append(q=qkv[:, :8], k=qkv[:, 8:10], v=qkv[:, 10:], q_out=qkv, k_out=None, pos=None)
    with pytest.raises(Taken):
        prompt(lse=torch.zeros(40), cu_k=i32(6))
    with pytest.raises(Taken):
        cached(lse=None, out=rows(6, 8))
    gb.attn_batch(i32(9), i32(3), i32(4, 2))


@pytest.mark.parametrize("bad", [
    dict(cu_q=i32(3)), dict(page_table=i32(2, 2)), dict(page_table=i32(3, 4)[:, :2]), dict(kv_len=i32(6)[::2]),
    dict(page_table=i32(3, 2).long()), dict(cu_q=i32(4).long()),
])
def test_batches_that_do_not_fit_are_refused(bad):
    with pytest.raises(ValueError):
        gb.attn_batch(**{**dict(cu_q=i32(4), kv_len=i32(3), page_table=i32(3, 2)), **bad})


@pytest.mark.parametrize("bad", [
    dict(v=POOL[:4]), dict(v=POOL[:, :1]), dict(k=POOL[:, :1], v=POOL[:, :1]), dict(k_scale=SCALE[:4]),
    dict(v_scale=SCALE[:, :1]), dict(v_scale=torch.zeros((5, 4), dtype=torch.uint8)[:, ::2]),
])
def test_caches_that_do_not_fit_are_refused(bad):
    with pytest.raises(ValueError):
        gb.attn_cache(**{**dict(k=POOL, v=POOL, k_scale=SCALE, v_scale=SCALE), **bad})


def test_rows_of_strided_heads_stay_refused():
    with pytest.raises(ValueError):
        attn._rows(rows(3, 2, 128)[:, :, ::2], 3, 2, 64)


def test_current_stream_without_the_undocumented_lookup(monkeypatch):
    class Current:
        cuda_stream = 1234
    monkeypatch.setattr(gb, "_current", None)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", Current)
    assert STREAM(None) == 1234
    assert STREAM(77) == 77 and STREAM(0) == 0
