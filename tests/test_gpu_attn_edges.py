"""Attention operators at the edges of their buffers and value ranges, each
element held to what its own sum can be off by."""
import numpy as np
import pytest
import torch

import attn_reference as ref
import paper_2607_12875_gb300 as gb
from test_gpu_attn import DT, U, Cache, attention_tolerance, cached_reference, i32, normal, prefix, wide

pytestmark = pytest.mark.gpu


def attention64(q, k, v, nq, nk, scale, causal=True, window=0):
    """Packed attention in 64 bits on the GPU: (out, size) with size = sum_j p_j |v_j| of each element."""
    out, size, a, b = [], [], 0, 0
    for n, m in zip(nq, nk):
        qs, ks, vs = q[a:a + n].double(), k[b:b + m].double(), v[b:b + m].double()
        a, b = a + n, b + m
        G = q.shape[1] // k.shape[1]
        ks, vs = ks.repeat_interleave(G, 1), vs.repeat_interleave(G, 1)
        pos = torch.arange(m - n, m, device=q.device)[:, None]
        j = torch.arange(m, device=q.device)[None, :]
        see = torch.ones((n, m), dtype=torch.bool, device=q.device)
        if causal:
            see &= j <= pos
        if window > 0:
            see &= j > pos - window
        s = torch.einsum("ihd,jhd->hij", qs, ks) * scale
        s = s.masked_fill(~see, -np.inf)
        top = s.amax(2, keepdim=True) if m else s.new_zeros((q.shape[1], n, 1))
        p = torch.exp(s - top.masked_fill(torch.isneginf(top), 0.0))
        p = p / p.sum(2, keepdim=True).masked_fill(~see.any(1)[None, :, None], 1.0)
        out.append(torch.einsum("hij,jhd->ihd", p, vs))
        size.append(torch.einsum("hij,jhd->ihd", p, vs.abs()))
    return torch.cat(out), torch.cat(size)


def bf16_bound(want, size):
    """The result's rounding to bf16 and the weights', each at most 2^-8 of itself; fp32 scores and exponentials."""
    return 1.05 * 2.0 ** -8 * (want.abs() + size) + 2e-5 * size


# ------------------------------------------------------------------- rotary


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_angles(layout):
    """cos and sin themselves (a pair of 1 and 0), near the multiples of a quarter turn, where one of them is small and has the
    angle's error alone: 2^-27 half turns (and 2^-32 turns cut off), beside two units in the last place (sincospif and
    the pair's 0 * sin)."""
    T, R = 200000, 32
    pos = np.random.default_rng(0).integers(-(1 << 20), 1 << 20, T)
    cfg = gb.attn_config(1, 1, R, act="f32", rotary_dim=R, rotary_layout=layout)
    x = torch.zeros((T, 1, R), device="cuda")
    first = np.arange(R // 2) if layout == "half" else 2 * np.arange(R // 2)
    x[:, 0, first] = 1.0
    y = torch.empty_like(x)
    gb.attn_rope(cfg, x, None, i32(pos), gb.attn_rope_table(R), y, None)
    turn = np.array([10000.0 ** (-2.0 * i / R) for i in range(R // 2)], dtype=np.longdouble) * pos[:, None].astype(np.longdouble)
    for got, want in ((wide(y)[:, 0, first], np.cos(turn)), (wide(y)[:, 0, first + (R // 2 if layout == "half" else 1)], np.sin(turn))):
        small = np.abs(want) < 0.1
        assert small.sum() > 10000
        err = np.abs(got - want)
        # (the table's entries: 2^-64 turns; frequencies in 64 bits: 2^-53 of up to 2^20 radians)
        assert (err <= np.pi * 2.0 ** -27 + 2 * np.pi * 2.0 ** -32 + 2.0 ** -22 * np.abs(want) + 2.0 ** -31)[small].all(), err[small].max()
        assert (err <= np.pi * 2.0 ** -27 + 2.0 ** -22).all()


# ------------------------------------------------------------------- append


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["act", "e4m3"])
@pytest.mark.parametrize("infinite", [False, True])
@pytest.mark.parametrize("page,D,R,new,lens", [
    (128, 128, 128, [300], [300]),                          # more tokens in a page than a block takes at a time
    (64, 256, 64, [100, 64], [130, 64]),
    (64, 64, 64, [13, 1, 1, 1], [13, 70, 1, 64]),           # few tokens a sequence on average: a warp's work, several passes
    (16, 128, 32, [13, 1, 1, 1], [40, 33, 1, 16]),
    (64, 64, 64, [40, 3], [40, 80]),                        # one pass
])
def test_append_in_place(act, kind, infinite, page, D, R, new, lens):
    """Rotated queries and keys over the ones that came: the cache holds what it holds with outputs of their own."""
    rng = np.random.default_rng(page + D)
    Hkv, G, T = 3, 2, sum(new)
    k, v, q = normal(rng, (T, Hkv, D), act), normal(rng, (T, Hkv, D), act), normal(rng, (T, Hkv * G, D), act)
    if infinite:  # in the scale's way, so that the maxima are searched again
        v[1, 0, 3], v[2, 2, D - 1] = float("inf"), float("-inf")
        if R < D:
            k[1, 1, D - 1] = float("inf")
    cfg = gb.attn_config(Hkv * G, Hkv, D, act=act, rotary_dim=R, rotary_scale=1.25, cache=kind, page=page)
    table = gb.attn_rope_table(R)
    caches = [Cache(np.random.default_rng(1), act, kind, Hkv, D, page, lens) for _ in range(2)]
    want = [caches[0].stored(w) for w in "kv"]
    keep = (prefix(new), i32(lens), caches[0].dev_table)
    outs = []
    for c, alias in zip(caches, (False, True)):
        kk, qq = k.clone(), q.clone()
        ko, qo = (kk, qq) if alias else (torch.empty_like(k), torch.empty_like(q))
        gb.attn_append(cfg, gb.attn_batch(*keep), kk, v, table, c.bundle, q=qq, q_out=qo, k_out=ko)
        outs.append([ko, qo, c.k, c.v] + ([c.ks, c.vs] if kind == "e4m3" else []))
    bits = {4: torch.int32, 2: torch.int16, 1: torch.uint8}
    for a, b in zip(*outs):
        assert torch.equal(a.view(bits[a.element_size()]), b.view(bits[b.element_size()]))
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(new, lens)])
    turned = ref.rotate(wide(k), pos, ref.frequencies(R), "half", 1.25)
    for which, (vals, exps), x in (("k", want[0], turned), ("v", want[1], wide(v))):
        ref.append(vals, exps, x, new, lens, caches[1].table, page)
        got, got_e = caches[1].stored(which)
        if exps is None:
            fin = np.isfinite(vals)
            assert np.array_equal(np.isfinite(got), fin)
            assert (np.abs(got[fin] - vals[fin]) <= U[act] * np.abs(vals[fin]) + 1e-6 * np.abs(vals[fin]).max()).all()
            continue
        assert np.array_equal(got_e, exps)
        # equal codes, but where fp32's rotation falls on the other side of a rounding boundary: then the next code
        differ = got != vals
        assert differ.mean() <= (1e-4 if which == "k" else 0.0)
        assert (np.abs(got - vals)[differ] <= np.abs(vals[differ]) / 8 + 2.0 ** -9).all()


# ------------------------------------------------------------------- cached


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_cached_scale_that_is_no_number_at_keys_unseen(act, D):
    """A page's scale byte of 255 (NaN) matters to the rows that see one of its keys alone."""
    rng = np.random.default_rng(D)
    page, n, lens = 16, [1, 3], [320, 194]
    c = Cache(rng, act, "e4m3", 2, D, page, lens)
    q = normal(rng, (4, 4, D), act)
    cfg = gb.attn_config(4, 2, D, act=act, window=100, cache="e4m3", page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 4, 2), dtype=torch.uint8, device="cuda")
    keep = (prefix(n), i32(lens), c.dev_table)
    # keys 192 .. 207: of the first sequence before its token's window (220 ..), in a block of 64 keys that it reaches
    # into; of the second one the tokens at 192 and 193 see some of them, the token at 191 none
    ids = [int(c.table[b, 12]) for b in range(2)]
    keep_scale = c.vs.clone()
    c.vs[ids] = 255
    out, lse = torch.zeros_like(q), torch.zeros((4, 4), device="cuda")
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws, lse=lse)
    got = wide(out)
    assert np.isnan(got[2:]).all() and torch.isfinite(lse).all()
    c.vs.copy_(keep_scale)
    want, _ = cached_reference(wide(q), c, n, lens, cfg.scale, True, 100)
    vmax = max(np.abs(c.rows("v", b, m)[0]).max() for b, m in enumerate(lens))
    assert (np.abs(got - want)[:2] <= attention_tolerance(act, want, vmax)[:2]).all()


def test_cached_many_small_weights_beside_a_large_one():
    """One key far ahead of all others, its value 0: the result is the sum of the others' small weights. The kernel's
    weights are fp16 and the largest is 2^9 or more, so each is off by 2^-11 of itself or 2^-34 of the largest; sums and
    scores by fp32's rounding."""
    for D, m in [(64, 192), (96, 192), (128, 192), (128, 40000)]:
        page = 64
        per = -(-m // page)
        k, v = (torch.zeros((per, 1, page, D), dtype=torch.uint8, device="cuda") for _ in range(2))
        ks, vs = (torch.full((per, 1), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        v.fill_(0x38)                      # 1.0
        k[0, 0, 0, 0], v[0, 0, 0] = 0x55, 0   # 13.0
        q = torch.zeros((1, 1, D), dtype=torch.bfloat16, device="cuda")
        q[0, 0, 0] = 1.4375
        cfg = gb.attn_config(1, 1, D, scale=1.0, cache="e4m3", page=page)
        ws = torch.zeros(gb.attn_workspace_size(cfg, 1, 1), dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(q)
        keep = (i32([0, 1]), i32([m]), i32(np.arange(per)[None]))
        gb.attn_cached(cfg, gb.attn_batch(*keep), q, gb.attn_cache(k, v, ks, vs), out, ws)
        w = np.exp(-13.0 * 1.4375)
        want = (m - 1) * w / (1 + (m - 1) * w)
        assert 2.0 ** -28 < w < 2.0 ** -26  # the test's premise
        bound = 1.05 * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -34 / w) * want + 2e-5 * want
        assert (np.abs(wide(out) - want) <= bound).all(), (D, m, float(out[0, 0, 0]), want)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["act", "e4m3"])
def test_cached_nan_values_of_no_weight(act, kind):
    """A value that is no number makes its column so for every row that sees it, however small its weight, whether it
    lies in the part of the keys that has the largest score or in another one."""
    D, page, m = 64, 64, 4096
    k, v = (torch.zeros((m // page, 1, page, D), dtype=torch.uint8 if kind == "e4m3" else torch.float32, device="cuda") for _ in range(2))
    scales = [torch.full((m // page, 1), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if kind == "e4m3" else [None] * 2
    one, nan = (0x38, 0x7f) if kind == "e4m3" else (1.0, float("nan"))
    k[:, 0, :, 0] = one                   # every key's score is q's first element, but
    k[m // page - 1, 0, 5, 1] = one       # one that is 300 ahead
    v.fill_(one)
    v[3, 0, 7, 20] = nan
    if kind == "act":
        k, v = k.to(DT[act]), v.to(DT[act])
    q = torch.zeros((1, 1, D), dtype=DT[act], device="cuda")
    q[0, 0, 0], q[0, 0, 1] = 1.0, 300.0
    cfg = gb.attn_config(1, 1, D, act=act, scale=1.0, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 1, 1), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    keep = (i32([0, 1]), i32([m]), i32(np.arange(m // page)[None]))
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, gb.attn_cache(k, v, *scales), out, ws)
    want = np.ones(D)
    want[20] = np.nan
    assert np.array_equal(wide(out)[0, 0], want, equal_nan=True)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["act", "e4m3"])
@pytest.mark.parametrize("m", [40, 3000])
def test_cached_scores_of_minus_infinity(act, kind, m):
    """A row that sees keys, all with scores of -inf, is 0 / 0 as the formula has it; a row whose keys have no page is 0."""
    rng = np.random.default_rng(m)
    D, page = 64, 16
    c = Cache(rng, act, kind, 1, D, page, [m, m])
    if kind == "act":
        c.k.abs_().clamp_(min=0.5)
    else:
        c.k.bitwise_and_(0x7f).clamp_(min=8)
    c.table[1] = -1
    c.table[0, 3:] = -1
    q = normal(rng, (2, 3, D), act)
    q[0, 1] = float("-inf")
    cfg = gb.attn_config(3, 1, D, act=act, cache=kind, page=page)
    ws = torch.zeros(gb.attn_workspace_size(cfg, 2, 2), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((2, 3), device="cuda")
    keep = (i32([0, 1, 2]), i32([m, m]), i32(c.table))
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws, lse=lse)
    got = wide(out)
    assert np.isnan(got[0, 1]).all() and np.isfinite(got[0, [0, 2]]).all() and (got[1] == 0).all()
    assert torch.isneginf(lse[0, 1]) and torch.isfinite(lse[0, 0]) and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("act,kind,D", [("bf16", "e4m3", 64), ("bf16", "e4m3", 96), ("bf16", "e4m3", 128), ("bf16", "act", 64),
                                        ("bf16", "act", 128), ("f32", "act", 64), ("f32", "e4m3", 80)])
@pytest.mark.parametrize("Hq,Hkv,n,lens", [(8, 1, [1, 1], [9000, 70]), (8, 2, [5, 1], [7001, 2500])])
def test_cached_long_contexts_element_by_element(act, kind, D, Hq, Hkv, n, lens):
    """The average of thousands of values is small beside the largest of them: each element is held to the sum that
    it is made of. Weights of 8 (bf16 cache) or 11 bits (e4m3), results of 8, fp32 scores and sums."""
    rng = np.random.default_rng(D + Hq)
    c = Cache(rng, act, kind, Hkv, D, 32, lens)
    q = normal(rng, (sum(n), Hq, D), act, 0.5)
    cfg = gb.attn_config(Hq, Hkv, D, act=act, cache=kind, page=32)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(n), len(n)), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    keep = (prefix(n), i32(lens), c.dev_table)
    gb.attn_cached(cfg, gb.attn_batch(*keep), q, c.bundle, out, ws)
    k, v = (torch.from_numpy(np.concatenate([c.rows(w, b, m)[0] for b, m in enumerate(lens)])).cuda() for w in "kv")
    want, size = attention64(q, k, v, n, lens, cfg.scale)
    weight, result = (2.0 ** -24, 2.0 ** -24) if act == "f32" else (2.0 ** -8 if kind == "act" else 2.0 ** -11, 2.0 ** -8)
    bound = 1.05 * (result * want.abs() + weight * size) + 2e-5 * size
    assert ((out.double() - want).abs() <= bound).all()
    assert gb.moe_device_status(ws) == gb.OK


# ------------------------------------------------------------------- prompt


@pytest.mark.parametrize("Hq,Hkv,D,nq,nk", [
    # more items than SMs, items without keys between the others; head sizes whose results leave in an odd number of pieces
    (400, 400, 96, [128, 128, 256, 130, 128], [128, 0, 100, 0, 256]),
    (400, 400, 32, [128, 128, 256, 130, 128], [128, 0, 100, 0, 256]),
    (800, 400, 80, [64, 64, 128, 64], [64, 0, 128, 0]),
    # so few that a tile's keys are dealt to both halves
    (20, 20, 64, [512, 512, 512, 512], [512, 0, 600, 0]),
    (20, 20, 96, [512, 512, 512, 512], [512, 0, 600, 0]),
    (20, 20, 32, [512, 512, 512, 512], [512, 0, 600, 0]),
])
def test_prompt_items_with_and_without_keys_in_turn(Hq, Hkv, D, nq, nk):
    rng = np.random.default_rng(D)
    q, k, v = (normal(rng, (sum(n), h, D), "bf16") for n, h in ((nq, Hq), (nk, Hkv), (nk, Hkv)))
    cfg = gb.attn_config(Hq, Hkv, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(nq), len(nq)), dtype=torch.uint8, device="cuda")
    want, size = attention64(q, k, v, nq, nk, cfg.scale)
    bound, cu_q, cu_k = bf16_bound(want, size), prefix(nq), prefix(nk)
    for _ in range(10):
        out = torch.full_like(q, float("nan"))
        gb.attn_prompt(cfg, q, k, v, cu_q, cu_k, out, ws)
        assert ((out.double() - want).abs() <= bound).all()
    assert gb.moe_device_status(ws) == gb.OK


def test_prompt_dealt_keys_of_ragged_ends():
    """Dealt keys, more items than SMs, tiles whose last rows no warp has and whose keys are all in one half."""
    rng = np.random.default_rng(1)
    nq, nk, H, D = [272, 260, 290, 272], [100, 260, 20, 272], 20, 64
    q, k, v = (normal(rng, (sum(n), H, D), "bf16") for n in (nq, nk, nk))
    cfg = gb.attn_config(H, H, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(nq), len(nq)), dtype=torch.uint8, device="cuda")
    want, size = attention64(q, k, v, nq, nk, cfg.scale)
    bound, cu_q, cu_k = bf16_bound(want, size), prefix(nq), prefix(nk)
    for _ in range(20):
        out = torch.full_like(q, float("nan"))
        gb.attn_prompt(cfg, q, k, v, cu_q, cu_k, out, ws)
        assert ((out.double() - want).abs() <= bound).all()
    assert gb.moe_device_status(ws) == gb.OK


def elapsed(call, n=3):
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    call()
    best = float("inf")
    for _ in range(n):
        torch.cuda.synchronize()
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("H,n", [(16, 3000), (2, 2500)])
def test_prompt_rows_that_see_a_nan_value_cost_no_more(H, n):
    """A value that is not a number at the first token: every row sees it and its column is NaN, in about the time of
    any other call."""
    rng = np.random.default_rng(n)
    D = 128
    q, k, v = (normal(rng, (n, H, D), "bf16") for _ in range(3))
    cfg = gb.attn_config(H, H, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
    cu, out = prefix([n]), torch.empty_like(q)
    call = lambda: gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)  # noqa: E731
    plain = elapsed(call)
    want, size = attention64(q, k, v, [n], [n], cfg.scale)
    v[0, 1, 70] = float("nan")
    took = elapsed(call)
    hit = torch.zeros_like(want, dtype=torch.bool)
    hit[:, 1, 70] = True
    assert torch.equal(torch.isnan(out), hit)
    assert ((out.double() - want).abs() <= bf16_bound(want, size))[~hit].all()
    assert gb.moe_device_status(ws) == gb.OK
    assert took <= 2 * plain + 0.1, (took, plain)


@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (200, 100), (168, 24)])
def test_prompt_rows_beside_values_they_do_not_see(Hq, Hkv, window):
    """Values that are no numbers at a token in the middle, one of them infinite, and in the rows behind the last
    sequence: rows that see them have them in their columns, all others are right (heads that are no power of two in a
    group, keys dealt to two halves, tiles of many items)."""
    rng = np.random.default_rng(window + Hq)
    D, nq = 64, [140, 260, 33]
    T = sum(nq)
    q, k, v = (normal(rng, (T + 40, h, D), "bf16") for h in (Hq, Hkv, Hkv))
    cfg = gb.attn_config(Hq, Hkv, D, window=window)
    ws = torch.zeros(gb.attn_workspace_size(cfg, T, 3), dtype=torch.uint8, device="cuda")
    want, size = attention64(q[:T], k[:T], v[:T], nq, nq, cfg.scale, window=window)
    v[T:] = float("nan")
    v[140 + 77, 1, 5] = float("nan")
    v[140 + 90, 0, 9] = float("inf")
    out = torch.empty_like(q)
    gb.attn_prompt(cfg, q, k, v, prefix(nq), prefix(nq), out, ws)
    hit, G = torch.zeros_like(want, dtype=torch.bool), Hq // Hkv
    end = lambda at: min(400, at + window if window else 400)  # noqa: E731
    hit[217:end(217), G:2 * G, 5] = True
    hit[230:end(230), :G, 9] = True
    assert torch.equal(~torch.isfinite(out[:T]), hit)
    assert ((out[:T].double() - want).abs() <= bf16_bound(want, size))[~hit].all()
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("H,n", [(16, 3000), (2, 2500)])
def test_prompt_ignores_what_lies_behind_the_end(H, n):
    """Keys and values in the rows behind the last sequence are no numbers."""
    rng = np.random.default_rng(n)
    D = 128
    q, k, v = (normal(rng, (n + 100, H, D), "bf16") for _ in range(3))
    cfg = gb.attn_config(H, H, D)
    ws = torch.zeros(gb.attn_workspace_size(cfg, n, 1), dtype=torch.uint8, device="cuda")
    want, size = attention64(q[:n], k[:n], v[:n], [n], [n], cfg.scale)
    v[n:], k[n:] = float("nan"), float("inf")
    cu, out = prefix([n]), torch.empty_like(q)
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    assert ((out[:n].double() - want).abs() <= bf16_bound(want, size)).all()
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("Hq,Hkv,D,n,window", [(8, 2, 128, [3001, 513], 0), (4, 4, 64, [2600], 700), (6, 2, 96, [1500, 900], 0)])
def test_prompt_long_rows_element_by_element(Hq, Hkv, D, n, window):
    rng = np.random.default_rng(D)
    q, k, v = (normal(rng, (sum(n), h, D), "bf16") for h in (Hq, Hkv, Hkv))
    cfg = gb.attn_config(Hq, Hkv, D, window=window)
    ws = torch.zeros(gb.attn_workspace_size(cfg, sum(n), len(n)), dtype=torch.uint8, device="cuda")
    out, cu = torch.zeros_like(q), prefix(n)
    gb.attn_prompt(cfg, q, k, v, cu, cu, out, ws)
    want, size = attention64(q, k, v, n, n, cfg.scale, window=window)
    assert ((out.double() - want).abs() <= bf16_bound(want, size)).all()
    assert gb.moe_device_status(ws) == gb.OK


# ------------------------------------------------------------------- strides


LAYOUTS = {
    "heads first": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1),
    "tokens apart by no multiple of a head": lambda t: torch.cat([t.flatten(1), t.new_zeros((t.shape[0], 24))], 1)[:, :t[0].numel()].view(t.shape),
    "heads wide apart": lambda t: torch.cat([t, t.new_zeros(t.shape)], 1).view(t.shape[0], 2, t.shape[1], t.shape[2])[:, 0],
}


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_layouts(act, layout):
    """Every operator on rows laid out otherwise gives what it gives on contiguous ones, bit for bit, and leaves its inputs alone."""
    rng = np.random.default_rng(12)
    Hq, Hkv, D, n = 6, 2, 64, [130, 77, 1]
    T, lay = sum(n), LAYOUTS[layout]
    q, k, v = normal(rng, (T, Hq, D), act), normal(rng, (T, Hkv, D), act), normal(rng, (T, Hkv, D), act)
    cfg = gb.attn_config(Hq, Hkv, D, act=act, rotary_dim=32, cache="e4m3", page=16)
    ws = torch.zeros(gb.attn_workspace_size(cfg, T, 3), dtype=torch.uint8, device="cuda")
    table, pos, cu = gb.attn_rope_table(32), i32(rng.integers(0, 999, T)), prefix(n)
    results = []
    for put in (lambda t: t.clone(), lay):
        a, b, c = put(q), put(k), put(v)
        outs = [put(torch.zeros_like(t)) for t in (q, k, q, k, q, q)]
        cache = Cache(np.random.default_rng(5), act, "e4m3", Hkv, D, 16, n)
        keep = (cu, i32(n), cache.dev_table)
        batch = gb.attn_batch(*keep)
        assert all(torch.equal(x, y) for x, y in zip((a, b, c), (q, k, v)))
        gb.attn_rope(cfg, a, b, pos, table, outs[0], outs[1])
        gb.attn_append(cfg, batch, b, c, table, cache.bundle, q=a, q_out=outs[2], k_out=outs[3])
        gb.attn_prompt(cfg, outs[2], outs[3], c, cu, cu, outs[4], ws)
        gb.attn_cached(cfg, batch, outs[2], cache.bundle, outs[5], ws)
        assert all(torch.equal(x, y) for x, y in zip((a, b, c), (q, k, v)))
        results.append([t.clone(memory_format=torch.contiguous_format) for t in outs] + [cache.k, cache.v, cache.ks, cache.vs])
    for x, y in zip(*results):
        assert torch.equal(x, y)
    assert gb.moe_device_status(ws) == gb.OK
