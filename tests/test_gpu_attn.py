"""Attention operators against their 64-bit forms: rotary positions, appending
to the cache, attention over packed prompts and over the cache."""
import numpy as np
import pytest
import torch

import attn_reference as ref
import paper_2607_12875_gb300 as gb

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative: significands of 24 and 8 bits


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


def normal(rng, shape, act, sigma=1.0):
    return torch.from_numpy((sigma * rng.standard_normal(shape)).astype(np.float32)).cuda().to(DT[act])


def strided(t):
    """The same values as rows of a wider buffer with other tensors' columns between (tokens and heads apart)."""
    T, H, D = t.shape
    buf = torch.full((T, H + 3, D + 16), float("nan"), dtype=t.dtype, device=t.device)
    buf[:, 1:H + 1, 8:D + 8] = t
    return buf[:, 1:H + 1, 8:D + 8]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prefix(v):
    return i32([0] + list(np.cumsum(v)))


# ------------------------------------------------------------------- rotary


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,D,R", [(1, 4, 1, 64, 64), (37, 6, 2, 128, 32), (130, 3, 3, 80, 48), (5, 1, 1, 256, 256),
                                          (700, 8, 2, 64, 0), (3000, 1, 1, 16, 16)])
def test_rope(act, layout, T, Hq, Hkv, D, R):
    rng = np.random.default_rng(T + D)
    q, k = normal(rng, (T, Hq, D), act), strided(normal(rng, (T, Hkv, D), act))
    # positions over the whole range: near 0, past 2^20, the largest int32, before the start
    pos = rng.integers(0, 1 << 20, T)
    pos[:3] = [2 ** 31 - 1, -5, 0][:min(3, T)]
    cfg = gb.attn_config(Hq, Hkv, D, act=act, rotary_dim=R, rotary_layout=layout, rotary_scale=1.25)
    table = gb.attn_rope_table(R, 10000.0) if R else None
    qo, ko = torch.empty_like(q), strided(torch.zeros_like(q[:, :Hkv]))
    gb.attn_rope(cfg, q, k, i32(pos), table, qo, ko)
    f = ref.frequencies(R) if R else np.zeros(0)
    for x, y in ((q, qo), (k, ko)):
        want = ref.rotate(wide(x), pos, f, layout, 1.25)
        # one rounding of the result; the angle to 2^-25 half turns, cos and sin and the two products in fp32; the
        # 64-bit reference's own angle at position 2^31 is good to 2^31 * 2^-53
        tol = U[act] * np.abs(want) + 1.25 * 6e-7 * np.abs(wide(x)).max()
        assert (np.abs(wide(y) - want) <= tol).all()
    # in place, and back
    q2 = q.clone()
    gb.attn_rope(cfg, q2, None, i32(pos), table, q2, None)
    assert torch.equal(q2, qo)
    gb.attn_rope(cfg, None, k, i32(pos), table, None, k)
    assert torch.equal(k, ko)
    plain = gb.attn_config(Hq, Hkv, D, act=act, rotary_dim=R, rotary_layout=layout)
    gb.attn_rope(plain, q, None, i32(pos), table, qo, None)
    gb.attn_rope(plain, qo, None, i32(pos), table, qo, None, inverse=True)
    assert (np.abs(wide(qo) - wide(q)) <= (3 * U[act] + 2e-6) * np.abs(wide(q)).max()).all()


def test_rope_scalings_change_the_angles():
    """linear: positions act divided; ntk and ramp keep the fastest pair and slow the slowest by the factor."""
    R, base = 128, 10000.0
    f = ref.frequencies(R, base)

    def freqs(**kw):
        t = gb.attn_rope_table(R, base, device="cpu", **kw).numpy().view(np.uint64)
        return t.astype(np.float64) / 2.0 ** 64 * 2 * np.pi
    assert np.allclose(freqs(), f, rtol=1e-12)
    assert np.allclose(freqs(scaling="linear", factor=4.0), f / 4, rtol=1e-12)
    ntk = freqs(scaling="ntk", factor=4.0)
    assert np.isclose(ntk[0], 1.0, rtol=1e-12) and np.isclose(ntk[-1], f[-1] / 4, rtol=1e-9)
    ramp = freqs(scaling="ramp", factor=8.0, original_ctx=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(ramp[turns > 40], f[turns > 40], rtol=1e-12)
    assert np.allclose(ramp[turns < 0.7], f[turns < 0.7] / 8, rtol=1e-12)
    assert (np.diff(ramp) < 0).all()


def test_rope_inverse_is_the_gradient():
    """d <w, rope(x)> / dx by central differences (the map is linear: exact but for rounding) is rope(w, inverse)."""
    rng = np.random.default_rng(3)
    T, H, D, R = 9, 2, 64, 32
    cfg = gb.attn_config(H, H, D, act="f32", rotary_dim=R, rotary_layout="interleaved", rotary_scale=1.1)
    table = gb.attn_rope_table(R)
    pos = i32(rng.integers(0, 3000, T))
    x, w = normal(rng, (T, H, D), "f32"), normal(rng, (T, H, D), "f32")
    g, y = torch.empty_like(x), torch.empty_like(x)
    gb.attn_rope(cfg, w, None, pos, table, g, None, inverse=True)
    for t, h, d in [(0, 0, 0), (3, 1, 7), (8, 1, 31), (5, 0, 32), (2, 1, 63)]:
        v = []
        for step in (0.5, -0.5):
            xs = x.clone()
            xs[t, h, d] += step
            gb.attn_rope(cfg, xs, None, pos, table, y, None)
            v.append(float((w.double() * y.double())[t, h].sum()))
        # fp32 sums of 64 terms of about 1
        assert abs(v[0] - v[1] - float(g[t, h, d])) <= 2e-5


# ------------------------------------------------------------------- append


class Cache:
    """A pool with random contents, its 64-bit copy, and a table of scattered pages."""

    def __init__(self, rng, act, kind, Hkv, D, page, lens, extra=2, poison=False):
        per = max(1, max(-(-max(n, 0) // page) for n in lens))
        used = [-(-max(n, 0) // page) for n in lens]
        n = sum(used) + extra
        order = rng.permutation(n)
        self.table = np.full((len(lens), per), -1, dtype=np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = order[at:at + u]
            at += u
        self.page, self.kind = page, kind
        shape = (n, Hkv, page, D)
        if kind == "act":
            self.k, self.v = normal(rng, shape, act), normal(rng, shape, act)
            self.ks = self.vs = None
        else:
            codes = rng.integers(0, 127, (2,) + shape) | (rng.integers(0, 2, (2,) + shape) << 7)
            self.k, self.v = (torch.from_numpy(c.astype(np.uint8)).cuda() for c in codes)
            exps = rng.integers(-9, -5, (2, n, Hkv))  # values up to 448 * 2^-6
            self.ks, self.vs = (torch.from_numpy((e + 127).astype(np.uint8)).cuda() for e in exps)
        if poison:  # what no sequence has written may be NaN
            written = np.zeros((n, page), dtype=bool)
            for b, m in enumerate(lens):
                for p in range(max(m, 0)):
                    written[self.table[b, p // page], p % page] = True
            free = torch.from_numpy(~written).cuda()[:, None, :, None]
            bad = float("nan") if kind == "act" else 0x7f
            for t in (self.k, self.v):
                t.masked_fill_(free, bad)
        self.bundle = gb.attn_cache(self.k, self.v, self.ks, self.vs)
        self.dev_table = i32(self.table)

    def stored(self, which):
        """(values or code values, exponents) in 64 bits."""
        t, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        if s is None:
            return wide(t), None
        return ref.e4m3_values()[t.cpu().numpy()], s.cpu().numpy().astype(np.int64) - 127

    def rows(self, which, b, m):
        """Sequence b's first m rows [m, Hkv, D] and which of them have a page."""
        vals, exps = self.stored(which)
        if exps is not None:
            vals = vals * 2.0 ** exps[:, :, None, None]
        p = np.arange(m)
        ids = self.table[b, p // self.page]
        ok = (ids >= 0) & (ids < vals.shape[0])
        return vals[np.where(ok, ids, 0), :, p % self.page], ok


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["act", "e4m3"])
@pytest.mark.parametrize("layout,page,D,R,new,lens", [
    ("half", 16, 64, 64, [1, 1, 1], [1, 17, 32]),               # single tokens: a fresh page, a second page, a page's last slot
    ("interleaved", 64, 128, 64, [70, 0, 3], [200, 64, 3]),     # over a page's end, nothing new, a whole sequence
    ("half", 128, 80, 48, [300, 5], [300, 131]),
    ("half", 32, 256, 0, [33], [40]),
    ("interleaved", 16, 8, 0, [40, 2], [41, 2]),
])
def test_append(act, kind, layout, page, D, R, new, lens):
    rng = np.random.default_rng(page + D)
    Hkv, G, T = 3, 2, sum(new)
    c = Cache(rng, act, kind, Hkv, D, page, lens)
    want_k, want_v = c.stored("k"), c.stored("v")
    k, v, q = strided(normal(rng, (T, Hkv, D), act)), normal(rng, (T, Hkv, D), act, 3.0), normal(rng, (T, Hkv * G, D), act)
    k[0] *= 40.0  # the scale of the first sequence's page grows
    cfg = gb.attn_config(Hkv * G, Hkv, D, act=act, rotary_dim=R, rotary_layout=layout, cache=kind, page=page)
    table = gb.attn_rope_table(R) if R else None
    batch_t = (prefix(new), i32(lens), c.dev_table)
    qo, ko = torch.empty_like(q), torch.zeros_like(v)
    gb.attn_append(cfg, gb.attn_batch(*batch_t), k, v, table, c.bundle, q=q, q_out=qo, k_out=ko)
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(new, lens)])
    f = ref.frequencies(R) if R else np.zeros(0)
    turned = ref.rotate(wide(k), pos, f, layout)
    for got, want in ((qo, ref.rotate(wide(q), pos, f, layout)), (ko, turned)):
        assert (np.abs(wide(got) - want) <= U[act] * np.abs(want) + 1e-6 * np.abs(want).max()).all()
    for which, want, x in (("k", want_k, turned), ("v", want_v, wide(v))):
        vals, exps = want
        ref.append(vals, exps, x, new, lens, c.table, page)
        got, got_e = c.stored(which)
        if exps is None:
            assert (np.abs(got - vals) <= U[act] * np.abs(vals) + 1e-6 * np.abs(vals).max()).all()
            continue
        assert np.array_equal(got_e, exps)
        # equal codes, but where fp32's rotation falls on the other side of a rounding boundary: then the next code
        differ = got != vals
        assert differ.mean() <= (1e-4 if which == "k" else 0.0)
        assert (np.abs(got - vals)[differ] <= np.abs(vals[differ]) / 8 + 2.0 ** -9).all()


def test_append_again_gives_the_same():
    """The same append twice leaves the cache as after the first (the old scale covers what it reads)."""
    rng = np.random.default_rng(0)
    c = Cache(rng, "bf16", "e4m3", 2, 64, 16, [21])
    k, v = normal(rng, (3, 2, 64), "bf16", 9.0), normal(rng, (3, 2, 64), "bf16")
    cfg = gb.attn_config(2, 2, 64, rotary_dim=64, cache="e4m3", page=16)
    keep = (prefix([3]), i32([21]), c.dev_table)
    once = None
    for _ in range(2):
        gb.attn_append(cfg, gb.attn_batch(*keep), k, v, gb.attn_rope_table(64), c.bundle)
        state = [t.clone() for t in (c.k, c.v, c.ks, c.vs)]
        if once is not None:
            assert all(torch.equal(a, b) for a, b in zip(once, state))
        once = state


def test_append_leaves_out_what_has_no_page():
    """Pages outside the pool, positions before 0 and beyond the table: not stored, q and k still turned; NaN and
    infinities do not reach the scale."""
    rng = np.random.default_rng(5)
    D, page = 64, 16
    c = Cache(rng, "f32", "e4m3", 1, D, page, [40, 16, 16, 16])
    table = c.table.copy()
    table[0, 1] = c.k.shape[0]  # one past the pool
    table[1, 0] = -3
    new, lens = [40, 2, 20, 4], [40, 16, 16, 60]  # 20 new tokens of 16: positions -4 ..; the last one's table ends at 48
    T = sum(new)
    k, v = normal(rng, (T, 1, D), "f32"), normal(rng, (T, 1, D), "f32")
    v[3, 0, 5], v[4, 0, 6] = float("nan"), float("-inf")
    before_k, before_v = c.stored("k"), c.stored("v")
    cfg = gb.attn_config(1, 1, D, act="f32", cache="e4m3", page=page)
    ko = torch.zeros_like(k)
    keep = (prefix(new), i32(lens), i32(table))
    gb.attn_append(cfg, gb.attn_batch(*keep), k, v, None, c.bundle, k_out=ko)
    assert torch.equal(ko, k)
    for which, (vals, exps), x in (("k", before_k, wide(k)), ("v", before_v, wide(v))):
        ref.append(vals, exps, x, new, lens, table, page)
        got, got_e = c.stored(which)
        assert np.array_equal(got_e, exps)
        assert np.array_equal(got, vals, equal_nan=True)


# ---------------------------------------------------------------- attention


def attention_tolerance(act, want, vmax):
    """bf16: the result's rounding, and the weights' rounding to bf16 (each at most 2^-8 of itself, their values at
    most vmax). fp32: sums of some thousand terms and exponentials of arguments up to about 30, errors of either sign."""
    if act == "f32":
        return 2e-5 * vmax + 0 * want
    return 1.05 * 2.0 ** -8 * (np.abs(want) + vmax) + 2e-5 * vmax


PROMPTS = [
    # Hq, Hkv, D, lengths of queries, lengths of keys (None: the same), causal, window
    (4, 4, 64, [1, 0, 7, 130], None, True, 0),
    (8, 2, 128, [257, 33, 129], None, True, 0),
    (6, 2, 128, [300], None, True, 0),              # three heads per kv head
    (2, 1, 128, [640, 128], None, True, 100),       # sliding window
    (4, 2, 64, [50, 200], [333, 200], True, 0),     # queries at the end of longer keys
    (2, 2, 64, [40, 3], [10, 0], True, 0),          # more queries than keys: the first ones see none
    (4, 1, 128, [100, 260], [300, 20], False, 0),   # not causal
    (2, 2, 128, [200], [400], False, 64),           # window without causal: keys after the position too
    (3, 1, 80, [140, 65], None, True, 0),           # head sizes between
    (2, 1, 8, [70], None, True, 0),
    (2, 2, 96, [260], None, True, 0),
    (2, 1, 256, [90, 20], None, True, 0),           # past 128: CUDA cores
    (2, 1, 200, [33], None, True, 0),
]


def packed_reference(q, k, v, nq, nk, scale, causal, window):
    outs, lses, a, b = [], [], 0, 0
    for n, m in zip(nq, nk):
        o, s = ref.attention(q[a:a + n], k[b:b + m], v[b:b + m], np.arange(m - n, m), scale, causal, window)
        outs.append(o), lses.append(s)
        a, b = a + n, b + m
    return np.concatenate(outs), np.concatenate(lses)


def check_attention(out, lse, want, want_lse, act, vmax):
    got = wide(out)
    assert np.isfinite(got).all()
    bad = np.abs(got - want) - attention_tolerance(act, want, vmax)
    assert bad.max() <= 0, f"over by {bad.max():.2e} at {np.unravel_index(bad.argmax(), bad.shape)}"
    empty = np.isneginf(want_lse)
    gl = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(gl), empty)
    # scores in fp32 from sums of up to 256 products, log sums of about 10
    assert (np.abs(gl[~empty] - want_lse[~empty]) <= 1e-4).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,D,nq,nk,causal,window", PROMPTS)
def test_prompt(act, Hq, Hkv, D, nq, nk, causal, window):
    rng = np.random.default_rng(D + len(nq))
    nk = nk or nq
    q, k, v = normal(rng, (sum(nq), Hq, D), act, 2.0), normal(rng, (sum(nk), Hkv, D), act), normal(rng, (sum(nk), Hkv, D), act)
    cfg = gb.attn_config(Hq, Hkv, D, act=act, causal=causal, window=window)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(nq), len(nq)), dtype=torch.uint8, device="cuda")
    out = strided(torch.zeros_like(q))
    lse = torch.full((sum(nq), Hq), float("nan"), device="cuda")
    gb.attn_prompt(cfg, strided(q), strided(k), strided(v), prefix(nq), prefix(nk), out, ws, lse=lse)
    want, want_lse = packed_reference(wide(q), wide(k), wide(v), nq, nk, cfg.scale, causal, window)
    check_attention(out, lse, want, want_lse, act, np.abs(wide(v)).max())
    assert gb.moe_device_status(ws) == gb.OK


MANY_HEADS = [
    # as above, with so many heads that each CTA takes several tiles of rows
    (160, 160, 64, [1, 0, 7, 130], None, True, 0),
    (512, 64, 64, [257, 33], None, True, 0),
    (192, 64, 128, [150], None, True, 0),           # three heads per kv head
    (256, 128, 64, [200, 128], None, True, 100),
    (256, 128, 64, [50, 100], [233, 100], True, 0),
    (256, 64, 64, [40, 3], [10, 0], True, 0),
    (256, 64, 64, [100, 60], [300, 20], False, 0),
    (384, 128, 80, [70, 65], None, True, 0),        # head sizes between
    (1024, 32, 32, [37], None, True, 0),            # 32 heads per kv head: a token fills a warp's rows
    (640, 16, 16, [37, 5], None, True, 0),          # 40: tiles of 8 of them
]


@pytest.mark.parametrize("Hq,Hkv,D,nq,nk,causal,window", MANY_HEADS)
def test_prompt_of_many_heads(Hq, Hkv, D, nq, nk, causal, window):
    test_prompt("bf16", Hq, Hkv, D, nq, nk, causal, window)


@pytest.mark.parametrize("Hq,Hkv,D,nq,nk,causal,window", [
    (168, 24, 64, [3, 1, 0, 40, 7, 18, 2, 25], None, True, 0),       # 7 heads per kv head: rows of 8
    (240, 40, 128, [9, 33, 1, 14, 60], None, True, 0),               # 6
    (150, 50, 80, [37, 5, 12, 70], None, True, 20),                  # 3
    (320, 16, 64, [3, 5, 11], [203, 5, 11], True, 0),                # 20 of 32 rows
])
def test_short_prompts_of_odd_groups(Hq, Hkv, D, nq, nk, causal, window):
    test_prompt("bf16", Hq, Hkv, D, nq, nk, causal, window)


@pytest.mark.parametrize("H", [2, 200])
def test_prompt_with_infinite_and_nan_scores(H):
    """Where every score of a row is not a number, or one is infinite, the row is not a number; rows before are right."""
    rng = np.random.default_rng(3)
    n, D = 300, 64
    for bad in (float("nan"), float("inf")):
        q, k, v = (normal(rng, (n, H, D), "bf16") for _ in range(3))
        q[280] = float("nan")
        k[290, :, 3] = bad
        cfg = gb.attn_config(H, H, D)
        ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(q)
        gb.attn_prompt(cfg, q, k, v, prefix([n]), prefix([n]), out, ws)
        got = wide(out)
        assert np.isnan(got[280]).all()
        right = [i for i in range(290) if i != 280]
        clean = q.clone()
        clean[280] = 0.0
        want, _ = packed_reference(wide(clean)[:290], wide(k)[:290], wide(v)[:290], [290], [290], cfg.scale, True, 0)
        tol = attention_tolerance("bf16", want, np.abs(wide(v)).max())
        assert (np.abs(got[right] - want[right]) <= tol[right]).all()
        if np.isnan(bad):
            assert np.isnan(got[290:]).all()


def test_waits_that_run_out_in_a_call_of_many_tiles(monkeypatch):
    rng = np.random.default_rng(10)
    n, H, D = 300, 200, 64
    q, k, v = (normal(rng, (n, H, D), "bf16") for _ in range(3))
    cfg = gb.attn_config(H, H, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
    cu, out = prefix([n]), torch.zeros_like(q)
    monkeypatch.setenv("GBMOE_TC_WAIT_LIMIT_NS", "0")
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.EDEVICE_TIMEOUT
    monkeypatch.delenv("GBMOE_TC_WAIT_LIMIT_NS")
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.OK
    want, _ = packed_reference(wide(q), wide(k), wide(v), [n], [n], cfg.scale, True, 0)
    assert (np.abs(wide(out) - want) <= attention_tolerance("bf16", want, np.abs(wide(v)).max())).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_prompt_of_many_sequences(act):
    """More sequences than a warp or a block looks at in one go, runs of empty ones, and a long one behind them."""
    rng = np.random.default_rng(7)
    nq = [int(v) for v in rng.integers(0, 9, 700)] + [0] * 70 + [260] + [0] * 30 + [1, 2]
    Hq, Hkv, D = 4, 2, 64
    q, k, v = normal(rng, (sum(nq), Hq, D), act), normal(rng, (sum(nq), Hkv, D), act), normal(rng, (sum(nq), Hkv, D), act)
    cfg = gb.attn_config(Hq, Hkv, D, act=act)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(nq), len(nq)), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.full((sum(nq), Hq), float("nan"), device="cuda")
    gb.attn_prompt(cfg, q, k, v, prefix(nq), prefix(nq), out, ws, lse=lse)
    want, want_lse = packed_reference(wide(q), wide(k), wide(v), nq, nq, cfg.scale, True, 0)
    check_attention(out, lse, want, want_lse, act, np.abs(wide(v)).max())
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prompt_ignores_what_no_query_sees(act, bad):
    """Keys and values of the sequence behind, and of later tokens of the same sequence, hold NaN or infinities."""
    rng = np.random.default_rng(1)
    H, D, n = 2, 64, [150, 90]
    q, k, v = (normal(rng, (240, H, D), act) for _ in range(3))
    k[150:], v[150:], q[150:] = bad, bad, bad
    k[140:150], v[140:150] = bad, bad  # the first sequence's last keys: seen by its last queries only
    cfg = gb.attn_config(H, H, D, act=act)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 240, 2), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    gb.attn_prompt(cfg, q, k, v, prefix(n), prefix(n), out, ws)
    want, _ = packed_reference(wide(q)[:140], wide(k)[:140], wide(v)[:140], [140], [140], cfg.scale, True, 0)
    got = wide(out)
    assert (np.abs(got[:140] - want) <= attention_tolerance(act, want, np.abs(wide(v)[:140]).max())).all()
    assert not np.isfinite(got[140:]).any()
    # a single value: its column alone is not a number, and only from its row on
    k, v = normal(rng, (240, H, D), act), normal(rng, (240, H, D), act)
    q = normal(rng, (240, H, D), act)
    v[77, 1, 5] = bad
    gb.attn_prompt(cfg, q, k, v, prefix(n), prefix(n), out, ws)
    got = wide(out)
    hit = np.zeros(got.shape, dtype=bool)
    hit[77:150, 1, 5] = True
    assert np.array_equal(~np.isfinite(got), hit)
    v[77, 1, 5] = 0.0
    want, _ = packed_reference(wide(q), wide(k), wide(v), n, n, cfg.scale, True, 0)
    tol = attention_tolerance(act, want, np.abs(wide(v)).max())
    assert (np.abs(got - want)[~hit] <= tol[~hit]).all()


CACHED = [
    # Hq, Hkv, D, page, query tokens of each sequence, keys, causal, window
    (4, 1, 64, 16, [1, 1, 1, 1], [1, 16, 17, 500], True, 0),
    (8, 1, 128, 64, [1, 1, 1], [0, 63, 1000], True, 0),          # no key at all
    (7, 1, 128, 128, [1], [3001], True, 0),                      # split over the keys
    (6, 2, 128, 32, [4, 1, 0, 3], [700, 31, 5, 3], True, 0),     # several tokens, none, a whole sequence
    (32, 2, 64, 64, [5, 2], [1025, 90], True, 0),                # more rows than a tile
    (2, 2, 64, 16, [40], [41], True, 0),
    (8, 2, 128, 64, [1, 2], [2000, 777], True, 128),             # sliding window
    (8, 2, 96, 16, [1, 3], [640, 100], True, 0),
    (4, 4, 64, 32, [6], [4], True, 0),                           # more queries than keys
    (4, 2, 128, 64, [3], [300], False, 0),
    (2, 1, 80, 16, [1, 2], [300, 70], True, 0),                  # head sizes of the CUDA-core kernel
    (3, 1, 256, 64, [1], [700], True, 0),
    (2, 2, 8, 16, [2], [33], True, 0),
]


def cached_reference(q, c, n, lens, scale, causal, window):
    outs, lses, at = [], [], 0
    for b, (nq, m) in enumerate(zip(n, lens)):
        k, ok = c.rows("k", b, m)
        v, _ = c.rows("v", b, m)
        o, s = ref.attention(q[at:at + nq], k, v, np.arange(m - nq, m), scale, causal, window, present=ok)
        outs.append(o), lses.append(s)
        at += nq
    return np.concatenate(outs), np.concatenate(lses)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["act", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,page,n,lens,causal,window", CACHED)
def test_cached(act, kind, Hq, Hkv, D, page, n, lens, causal, window):
    rng = np.random.default_rng(D + page)
    c = Cache(rng, act, kind, Hkv, D, page, lens, poison=True)
    q = normal(rng, (sum(n), Hq, D), act, 2.0 if kind == "act" else 1.0)
    cfg = gb.attn_config(Hq, Hkv, D, act=act, causal=causal, window=window, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(n), len(n)), dtype=torch.uint8, device="cuda")
    out, lse = strided(torch.zeros_like(q)), torch.full((sum(n), Hq), float("nan"), device="cuda")
    keep = (prefix(n), i32(lens), c.dev_table)
    gb.attn_cached(cfg, gb.attn_batch(*keep), strided(q), c.bundle, out, ws, lse=lse)
    want, want_lse = cached_reference(wide(q), c, n, lens, cfg.scale, causal, window)
    vmax = max([np.abs(c.rows("v", b, m)[0]).max() for b, m in enumerate(lens) if m > 0])
    check_attention(out, lse, want, want_lse, act, vmax)
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act,kind,D", [("bf16", "e4m3", 64), ("bf16", "act", 128), ("f32", "act", 64)])
def test_cached_of_many_sequences(act, kind, D):
    """More sequences than a block looks at in one go, some without tokens or keys, one with most of the keys."""
    rng = np.random.default_rng(11)
    lens = [int(v) for v in rng.integers(0, 70, 600)] + [3000] + [int(v) for v in rng.integers(0, 70, 50)]
    n = [int(v) for v in rng.integers(0, 3, len(lens))]
    Hq, Hkv, page = 4, 2, 16
    c = Cache(rng, act, kind, Hkv, D, page, lens)
    q = normal(rng, (sum(n), Hq, D), act)
    cfg = gb.attn_config(Hq, Hkv, D, act=act, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(n), len(n)), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.full((sum(n), Hq), float("nan"), device="cuda")
    keep = (prefix(n), i32(lens), c.dev_table)
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws, lse=lse)
    want, want_lse = cached_reference(wide(q), c, n, lens, cfg.scale, True, 0)
    vmax = max([np.abs(c.rows("v", b, m)[0]).max() for b, m in enumerate(lens) if m > 0])
    check_attention(out, lse, want, want_lse, act, vmax)
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("kind", ["act", "e4m3"])
def test_cached_values_of_very_different_scales(kind):
    """A row that attends to a page of tiny values keeps their relative accuracy beside pages of large ones."""
    rng = np.random.default_rng(2)
    D, page, m = 64, 16, 64
    c = Cache(rng, "bf16", kind, 1, D, page, [m])
    tiny = int(c.table[0, 2])
    if kind == "e4m3":
        c.vs[tiny] = 127 - 9 - 24
        c.ks[tiny] = 127 - 6
    else:
        c.v[tiny] *= 2.0 ** -24
    q = torch.zeros((1, 1, D), device="cuda")
    row = c.rows("k", 0, m)[0][37, 0]
    q[0, 0] = torch.from_numpy((row / (row @ row) * 400.0).astype(np.float32)).cuda()  # key 37 (that page) far ahead
    q = q.to(torch.bfloat16)
    cfg = gb.attn_config(1, 1, D, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 1, 1), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    keep = (prefix([1]), i32([m]), c.dev_table)
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws)
    want, _ = cached_reference(wide(q), c, [1], [m], cfg.scale, True, 0)
    v37 = np.abs(c.rows("v", 0, m)[0][37]).max()
    assert np.abs(want).max() <= 1.01 * v37  # the test's premise: nothing else is seen
    assert (np.abs(wide(out) - want) <= attention_tolerance("bf16", want, v37)).all()


@pytest.mark.parametrize("act,kind,D", [("bf16", "e4m3", 128), ("bf16", "act", 64), ("f32", "e4m3", 64)])
def test_cached_masks_pages_outside_the_pool_and_later_tokens(act, kind, D):
    """Tokens without a page are masked; a NaN value that only the last query sees reaches that one alone."""
    rng = np.random.default_rng(8)
    page, n, lens = 16, [3, 1, 1], [200, 90, 40]
    c = Cache(rng, act, kind, 2, D, page, lens, poison=True)
    c.table[0, 4], c.table[1, 1] = -1, c.k.shape[0]
    c.table[2] = -1  # no page at all: as if there were no keys
    pg = int(c.table[0, 199 // page])
    if kind == "act":
        c.v[pg, :, 199 % page] = float("nan")
    else:
        c.v[pg, :, 199 % page] = 0xff
    q = normal(rng, (5, 4, D), act)
    cfg = gb.attn_config(4, 2, D, act=act, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 5, 3), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    keep = (prefix(n), i32(lens), i32(c.table))
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws)
    got = wide(out)
    assert np.isnan(got[2]).all() and (got[4] == 0).all()
    if kind == "act":
        c.v[pg, :, 199 % page] = 0.0
    else:
        c.v[pg, :, 199 % page] = 0
    want, _ = cached_reference(wide(q), c, n, lens, cfg.scale, True, 0)
    vmax = np.nanmax(np.abs(np.concatenate([c.rows("v", b, m)[0] for b, m in enumerate(lens)])))
    rows = [0, 1, 3]
    assert (np.abs(got[rows] - want[rows]) <= attention_tolerance(act, want[rows], vmax)).all()


@pytest.mark.parametrize("act,kind", [("bf16", "e4m3"), ("bf16", "act")])
def test_pool_past_32_bit_offsets(act, kind):
    """Pages whose elements lie past 2^31 (and, e4m3, past 2^32): appended to and read."""
    rng = np.random.default_rng(4)
    D, page, Hkv = 128, 128, 8
    n_pages = (1 << 32) // (Hkv * page * D) + 40 if kind == "e4m3" else (1 << 31) // (Hkv * page * D) + 40
    dt = torch.uint8 if kind == "e4m3" else torch.bfloat16
    pool = [torch.zeros((n_pages, Hkv, page, D), dtype=dt, device="cuda") for _ in range(2)]
    scale = [torch.full((n_pages, Hkv), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if kind == "e4m3" else [None, None]
    m = 300
    table = np.array([[n_pages - 1, n_pages - 30, 3]], dtype=np.int32)
    q, k, v = (normal(rng, (m, h, D), act) for h in (Hkv, Hkv, Hkv))
    cfg = gb.attn_config(Hkv, Hkv, D, act=act, cache=kind, page=page)
    bundle = gb.attn_cache(pool[0], pool[1], scale[0], scale[1])
    keep = (prefix([m]), i32([m]), i32(table), prefix([2]))
    gb.attn_append(cfg, gb.attn_batch(*keep[:3]), k, v, None, bundle)
    out = torch.zeros_like(q[:2])
    ws = torch.zeros(gb.attn_workspace_size(cfg, 2, 1), dtype=torch.uint8, device="cuda")
    gb.attn_cached(cfg, gb.attn_batch(keep[3], keep[1], keep[2]), q[-2:], bundle, out, ws)
    # against the stored values, gathered
    p = np.arange(m)

    def rows(i):
        x = pool[i][torch.from_numpy(table[0, p // page]).long().cuda(), :, torch.from_numpy(p % page).cuda()]
        if kind == "act":
            return wide(x)
        e = scale[i].cpu().numpy().astype(np.int64)[table[0, p // page]] - 127
        return ref.e4m3_values()[x.cpu().numpy()] * 2.0 ** e[:, :, None]
    want, _ = ref.attention(wide(q[-2:]), rows(0), rows(1), np.array([m - 2, m - 1]), cfg.scale)
    # the stored values are the appended ones to a code's rounding (3 bits of mantissa)
    assert np.abs(rows(0) - wide(k)).max() <= (0.0 if kind == "act" else np.abs(wide(k)).max() / 16)
    assert (np.abs(wide(out) - want) <= attention_tolerance(act, want, np.abs(rows(1)).max())).all()


def test_prompt_then_decode_on_another_stream():
    """A prompt is appended (8-bit cache) and attended, then decoded a token at a time, all on a side stream, and the
    last prompt row from the cache is near the one from the bf16 keys."""
    rng = np.random.default_rng(6)
    Hq, Hkv, D, n = 8, 2, 128, 77
    s = torch.cuda.Stream()
    cfg = gb.attn_config(Hq, Hkv, D, rotary_dim=D, cache="e4m3", page=32)
    c = Cache(rng, "bf16", "e4m3", Hkv, D, 32, [n + 4])
    table = gb.attn_rope_table(D)
    q, k, v = (normal(rng, (n + 4, h, D), "bf16") for h in (Hq, Hkv, Hkv))
    ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
    qr, kr, out, again = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(q)
    keep = [(prefix([n]), i32([n]))] + [(prefix([1]), i32([n + i + 1])) for i in range(4)]
    batches = [gb.attn_batch(a, b, c.dev_table) for a, b in keep]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        gb.attn_append(cfg, batches[0], k[:n], v[:n], table, c.bundle, q=q[:n], q_out=qr[:n], k_out=kr[:n])
        gb.attn_prompt(cfg, qr[:n], kr[:n], v[:n], keep[0][0], keep[0][0], out[:n], ws)
        gb.attn_cached(cfg, batches[0], qr[:n], c.bundle, again[:n], ws)
        for i in range(4):
            t = slice(n + i, n + i + 1)
            gb.attn_append(cfg, batches[1 + i], k[t], v[t], table, c.bundle, q=q[t], q_out=qr[t], k_out=kr[t])
            gb.attn_cached(cfg, batches[1 + i], qr[t], c.bundle, out[t], ws)
    s.synchronize()
    pos = np.arange(n + 4)
    f = ref.frequencies(D)
    qw, kw = ref.rotate(wide(q), pos, f, "half"), ref.rotate(wide(k), pos, f, "half")
    want, _ = ref.attention(qw, kw, wide(v), pos, cfg.scale)
    vmax = np.abs(wide(v)).max()
    # prompt rows: rotated q and k rounded to bf16 (scores off by some 2^-8 of about 3); cached rows: codes of 2^-4
    assert np.abs(wide(out)[:n] - want[:n]).max() <= 0.03 * vmax
    assert np.abs(wide(out)[n:] - want[n:]).max() <= 0.08 * vmax
    assert np.abs(wide(again)[:n] - want[:n]).max() <= 0.15 * vmax


def test_waits_that_run_out_are_reported_and_leave_the_next_call_clean(monkeypatch):
    """With a limit of 0 ns on the pipeline waits attn_prompt gives up, the error word says so, and a call with the
    normal limit is right again."""
    rng = np.random.default_rng(9)
    n, Hq, Hkv, D = 700, 4, 2, 128
    q, k, v = (normal(rng, (n, h, D), "bf16") for h in (Hq, Hkv, Hkv))
    cfg = gb.attn_config(Hq, Hkv, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
    cu, out = prefix([n]), torch.zeros_like(q)
    monkeypatch.setenv("GBMOE_TC_WAIT_LIMIT_NS", "0")
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.EDEVICE_TIMEOUT
    monkeypatch.delenv("GBMOE_TC_WAIT_LIMIT_NS")
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.OK
    want, _ = packed_reference(wide(q), wide(k), wide(v), [n], [n], cfg.scale, True, 0)
    assert (np.abs(wide(out) - want) <= attention_tolerance("bf16", want, np.abs(wide(v)).max())).all()
