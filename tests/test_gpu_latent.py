"""Latent attention against its 64-bit forms: appending to the cache, packed
prompts in the expanded form, cached tokens in the absorbed form."""
import numpy as np
import pytest
import torch

import attn_reference
import latent_reference as ref
import paper_2607_12875_gb300 as gb
from latent_reference import DT, U, Pool, apart, check, heads_first, i32, normal, prefix

pytestmark = pytest.mark.gpu


def workspace(cfg, T, B):
    return torch.zeros(gb.latent_workspace_size(cfg, T, B), dtype=torch.uint8, device="cuda")


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------- append


def appended64(cfg, kv, gamma, q, pos, layout):
    """Rows and queries after norm and rotation, in 64 bits."""
    R, P = cfg.latent_dim, cfg.rope_dim
    c = wide(kv)[:, :R]
    if gamma is not None:
        c = c / np.sqrt((c * c).mean(1, keepdims=True) + cfg.norm_eps) * wide(gamma)
    f = attn_reference.frequencies(P) if P else np.zeros(0)
    key = attn_reference.rotate(wide(kv)[:, None, R:], pos, f, layout, cfg.rotary_scale)[:, 0]
    turned = None if q is None else attn_reference.rotate(wide(q), pos, f, layout, cfg.rotary_scale)
    return np.concatenate((c, key), 1), turned


def close(got, want, act):
    """One rounding, and fp32 arithmetic on values up to the row's largest (angles: 1.2e-7 radians of two terms)."""
    top = np.abs(want).max(-1, keepdims=True)
    assert (np.abs(wide(got) - want) <= U[act] * np.abs(want) + 1e-6 * top).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("layout,page,R,P,H,norm,new,lens", [
    ("half", 16, 512, 64, 5, True, [1, 1, 1], [1, 17, 32]),            # single tokens: a fresh page, a second, a page's last slot
    ("interleaved", 64, 512, 64, 128, True, [70, 0, 3], [200, 64, 3]),  # over a page's end, nothing new, a whole sequence
    ("half", 128, 256, 32, 1, False, [300, 5], [300, 131]),
    ("interleaved", 32, 8, 128, 3, True, [33], [40]),
    ("half", 16, 504, 0, 0, True, [40, 2], [41, 2]),                    # nothing turns
    ("interleaved", 16, 264, 48, 7, True, [1] * 70, list(range(1, 71))),  # more sequences than a warp has lanes
    ("interleaved", 64, 512, 64, 16, True, [1400, 200], [1400, 1000]),    # several tokens a block
])
def test_append(act, layout, page, R, P, H, norm, new, lens):
    T, W = sum(new), R + P
    pool = Pool(page + R, act, W, page, lens)
    kv, gamma = apart(normal(1, (T, W), act, 3.0)), normal(2, (R,), act) if norm else None
    q = apart(normal(3, (T, H, P), act)) if H and P else None
    cfg = gb.latent_config(max(H, 1), latent_dim=R, rope_dim=P, act=act, rotary_layout=layout, rotary_scale=1.25, page=page)
    table = gb.attn_rope_table(P) if P else None
    keep = (prefix(new), i32(lens), i32(pool.table))
    before = pool.rows.clone()
    q_out = apart(torch.zeros_like(q)) if q is not None else None
    kv_out = apart(torch.zeros_like(kv))
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, table, gb.latent_cache(pool.rows), q=q, q_out=q_out, kv_out=kv_out)
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(new, lens)])
    rows, turned = appended64(cfg, kv, gamma, q, pos, layout)
    close(kv_out, rows, act)
    if q is not None:
        close(q_out, turned, act)
    # the cache: the same rows bit for bit in their slots, everything else as it was
    at = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        for p in range(m - n, m):
            before[pool.table[b, p // page], p % page] = kv_out[at]
            at += 1
    bits = torch.int32 if act == "f32" else torch.int16
    assert torch.equal(pool.rows.view(bits), before.view(bits))
    # in place, and without the optional outputs: the same
    kv2, rows2 = kv.clone(), pool.rows.clone()
    q2 = q.clone() if q is not None else None
    gb.latent_append(cfg, gb.attn_batch(*keep), kv2, gamma, table, gb.latent_cache(rows2), q=q2, q_out=q2, kv_out=kv2)
    assert torch.equal(kv2, kv_out) and (q is None or torch.equal(q2, q_out))
    assert torch.equal(rows2.view(bits), before.view(bits))
    rows3 = torch.zeros_like(pool.rows)
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, table, gb.latent_cache(rows3))
    assert torch.equal(torch.nan_to_num(rows2).where(rows3 != 0, 0), rows3)


def test_append_leaves_out_what_has_no_place():
    """Pages outside the pool, positions before 0 and beyond the table: not stored, outputs written all the same;
    tokens of no sequence: nothing is written. Positions of the caller turn, the place in the sequence stores."""
    page, R, P, H = 16, 64, 32, 2
    new, lens = [40, 2, 20, 4], [40, 16, 16, 60]
    pool = Pool(0, "f32", R + P, page, [40, 16, 16, 48], poison=False)
    pool.table[0, 1], pool.table[1, 0] = pool.rows.shape[0], -3
    T = sum(new) + 5  # five rows behind the last sequence, two before the first
    cu = prefix(new) + 2
    T += 2
    kv, gamma, q = normal(1, (T, R + P), "f32"), normal(2, (R,), "f32"), normal(3, (T, H, P), "f32")
    cfg = gb.latent_config(H, latent_dim=R, rope_dim=P, act="f32", page=page)
    before = pool.rows.clone()
    kv_out, q_out = torch.full_like(kv, 7.0), torch.full_like(q, 7.0)
    given = np.random.default_rng(0).integers(-5, 1 << 20, T)
    keep = (cu, i32(lens), i32(pool.table))
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, gb.attn_rope_table(P), gb.latent_cache(pool.rows), q=q, q_out=q_out,
                     kv_out=kv_out, positions=i32(given))
    rows, turned = appended64(cfg, kv, gamma, q, given, "interleaved")
    mine = slice(2, T - 5)
    close(kv_out[mine], rows[mine], "f32")
    close(q_out[mine], turned[mine], "f32")
    for t in (kv_out, q_out):
        assert (t[:2] == 7.0).all() and (t[T - 5:] == 7.0).all()
    at = 2
    for b, (n, m) in enumerate(zip(new, lens)):
        for p in range(m - n, m):
            if 0 <= p < 48 and 0 <= pool.table[b, p // page] < pool.rows.shape[0]:
                before[pool.table[b, p // page], p % page] = kv_out[at]
            at += 1
    assert torch.equal(pool.rows, before)


def test_append_of_values_that_are_no_numbers():
    """They stay in their token."""
    cfg = gb.latent_config(1, latent_dim=128, rope_dim=16, page=16)
    kv, gamma = normal(0, (3, 144), "bf16"), normal(1, (128,), "bf16")
    kv[1, 5], kv[1, 140] = float("nan"), float("inf")
    pool = torch.zeros((1, 16, 144), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(kv)
    keep = (prefix([3]), i32([3]), i32([[0]]))
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, gb.attn_rope_table(16), gb.latent_cache(pool), kv_out=out)
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all()
    assert torch.isnan(out[1, :128]).all() and torch.isfinite(out[1, 128:140]).all()
    assert torch.equal(torch.nan_to_num(pool[0, :3]), torch.nan_to_num(out))


# ------------------------------------------------------------------- expanded


PROMPTS = [
    # heads, N, P, V, lengths of queries, lengths of keys (None: the same), causal
    (4, 128, 64, 128, [1, 0, 7, 130], None, True),
    (3, 128, 64, 128, [257, 33, 129], None, True),
    (2, 128, 64, 128, [640, 128], None, True),
    (2, 128, 64, 128, [50, 200], [333, 200], True),     # queries at the end of longer keys
    (2, 128, 64, 128, [40, 3], [10, 0], True),          # more queries than keys: the first ones see none
    (4, 128, 64, 128, [100, 260], [300, 20], False),    # not causal
    (200, 128, 64, 128, [140, 5], None, True),          # more tiles than SMs
    (5, 64, 64, 64, [300], None, True),
    (3, 96, 64, 96, [140, 65], None, True),
    (2, 64, 32, 128, [260], None, True),
    (2, 24, 16, 40, [70, 200], None, True),
    (2, 128, 0, 128, [150], None, True),                # no rotary elements
    (2, 128, 128, 128, [90, 20], None, True),           # wider than the tensor cores' form
    (1, 8, 0, 8, [33], None, False),
]


def prompt_inputs(seed, act, H, N, P, V, nq, nk):
    Tq, Tk = sum(nq), sum(nk)
    q, k, v = normal(seed, (Tq, H, N + P), act, 1.5), normal(seed + 1, (Tk, H, N), act), normal(seed + 2, (Tk, H, V), act)
    return q, k, normal(seed + 3, (Tk, P), act) if P else None, v


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("H,N,P,V,nq,nk,causal", PROMPTS)
def test_prompt(act, H, N, P, V, nq, nk, causal):
    nk = nk or nq
    q, k, kr, v = prompt_inputs(N + len(nq), act, H, N, P, V, nq, nk)
    cfg = gb.latent_config(H, rope_dim=P, nope_dim=N, value_dim=V, act=act, causal=causal)
    ws = workspace(cfg, sum(nq), len(nq))
    want = ref.expanded(q, k, kr, v, nq, nk, cfg.scale, causal)
    for lay in (lambda t: t, apart, lambda t: heads_first(t) if t.dim() == 3 else apart(t)):
        out = lay(torch.full((sum(nq), H, V), float("nan"), dtype=DT[act], device="cuda"))
        lse = torch.full((sum(nq), H), float("nan"), device="cuda")
        gb.latent_prompt(cfg, lay(q), lay(k), lay(kr) if P else None, lay(v), prefix(nq), prefix(nk), out, ws, lse=lse)
        check(out, lse, want, act)
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_prompt_of_many_sequences(act):
    """More sequences than a block has threads, most of them short or empty, and rows around them left as they were."""
    rng = np.random.default_rng(7)
    lens = [int(x) for x in rng.choice([0, 1, 2, 5, 40], 700)]
    T, H = sum(lens), 2
    q, k, kr, v = prompt_inputs(3, act, H, 128, 64, 128, [T + 9], [T + 9])
    cfg = gb.latent_config(H, act=act)
    ws = workspace(cfg, T + 9, len(lens))
    out = torch.full((T + 9, H, 128), 7.0, dtype=DT[act], device="cuda")
    cu = prefix(lens) + 4
    gb.latent_prompt(cfg, q, k, kr, v, cu, cu, out, ws)
    cut = slice(4, T + 4)
    check(out[cut], None, ref.expanded(q[cut], k[cut], kr[cut], v[cut], lens, lens, cfg.scale), act)
    assert (out[:4] == 7.0).all() and (out[T + 4:] == 7.0).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_prompt_ignores_what_no_query_sees(act, bad):
    """Rows between and behind the sequences hold what is no number; so do a key and a value inside one of them,
    which reach the queries that see them and no others."""
    lens, H = [100, 37, 129], 2
    T = sum(lens)
    q, k, kr, v = prompt_inputs(11, act, H, 128, 64, 128, [T + 30], [T + 30])
    cfg = gb.latent_config(H, act=act)
    ws = workspace(cfg, T + 30, 3)
    for t in (k, kr, v):
        t[T:] = bad
    want = ref.expanded(q[:T], k[:T], kr[:T], v[:T], lens, lens, cfg.scale)
    out = torch.full((T, H, 128), 7.0, dtype=DT[act], device="cuda")
    gb.latent_prompt(cfg, q[:T], k, kr, v, prefix(lens), prefix(lens), out, ws)
    check(out, None, want, act)
    v[50, 1, 3] = bad                                   # a value at position 50 of the first sequence
    out2 = torch.full_like(out, 7.0)
    gb.latent_prompt(cfg, q[:T], k, kr, v, prefix(lens), prefix(lens), out2, ws)
    seen = torch.zeros_like(out, dtype=torch.bool)
    seen[50:100, 1, 3] = True
    assert not torch.isfinite(out2[seen]).any()
    check(torch.where(seen, out, out2), None, want, act)
    kr[120] = bad                                       # a key at position 20 of the second
    gb.latent_prompt(cfg, q[:T], k, kr, v, prefix(lens), prefix(lens), out2, ws)
    rows = torch.zeros_like(out, dtype=torch.bool)
    rows[120:137] = True
    assert torch.isnan(out2[rows]).any(-1).all() if bad != bad else True
    check(torch.where(seen | rows, out, out2), None, want, act)


@pytest.mark.parametrize("H,lens", [(4, [700]), (100, [300, 200])])   # keys dealt to both tiles; each CTA takes several items
def test_prompt_waits_that_run_out(monkeypatch, H, lens):
    """With a limit of 0 ns on the pipeline waits a call gives up, the error word says so, and the next is right again."""
    T = sum(lens)
    q, k, kr, v = prompt_inputs(13, "bf16", H, 128, 64, 128, lens, lens)
    cfg = gb.latent_config(H)
    ws, cu, out = workspace(cfg, T, len(lens)), prefix(lens), torch.zeros((T, H, 128), dtype=torch.bfloat16, device="cuda")
    monkeypatch.setenv("GBMOE_TC_WAIT_LIMIT_NS", "0")
    gb.latent_prompt(cfg, q, k, kr, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.EDEVICE_TIMEOUT
    monkeypatch.delenv("GBMOE_TC_WAIT_LIMIT_NS")
    gb.latent_prompt(cfg, q, k, kr, v, cu, cu, out, ws)
    assert gb.moe_device_status(ws) == gb.OK
    check(out, None, ref.expanded(q, k, kr, v, lens, lens, cfg.scale), "bf16")


# ------------------------------------------------------------------- absorbed


CACHED = [
    # heads, R, P, page, query tokens, keys, causal
    (128, 512, 64, 64, [1, 1, 1], [1, 300, 129], True),
    (16, 512, 64, 16, [4, 1, 3], [1000, 1, 2], True),     # more queries than keys
    (1, 512, 64, 32, [1, 1], [127, 128], True),
    (56, 512, 64, 128, [1, 2], [385, 640], True),
    (20, 512, 64, 64, [1, 0, 2, 1], [70, 50, 0, 64], True),  # a sequence without queries, one without keys
    (5, 256, 32, 16, [3, 1], [200, 17], False),
    (64, 384, 64, 64, [1], [5000], True),
    (24, 128, 16, 32, [2, 2, 2], [97, 33, 256], True),
    (32, 512, 0, 64, [1, 1], [100, 65], True),
    (12, 64, 16, 16, [1, 2], [50, 90], True),             # narrower than the tensor cores' form
    (3, 504, 128, 64, [1, 1], [333, 12], True),
    (128, 512, 64, 64, [7], [500], True),
]


def cached_case(seed, act, H, R, P, page, nq, lens, causal=True, sigma=1.0):
    pool = Pool(seed, act, R + P, page, lens)
    q = normal(seed + 5, (sum(nq), H, R + P), act, sigma)
    cfg = gb.latent_config(H, latent_dim=R, rope_dim=P, act=act, causal=causal, page=page)
    return pool, q, cfg


def run_cached(cfg, pool, q, nq, lens, out=None, lse=None, ws=None):
    if out is None:
        out = torch.full((q.shape[0], cfg.heads, cfg.latent_dim), float("nan"), dtype=q.dtype, device="cuda")
    keep = (prefix(nq), i32(lens), i32(pool.table))
    ws = workspace(cfg, q.shape[0], len(nq)) if ws is None else ws
    gb.latent_cached(cfg, gb.attn_batch(*keep), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
    assert gb.moe_device_status(ws) == gb.OK
    return out


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("H,R,P,page,nq,lens,causal", CACHED)
def test_cached(act, H, R, P, page, nq, lens, causal):
    pool, q, cfg = cached_case(R + H, act, H, R, P, page, nq, lens, causal)
    want = ref.absorbed(q, pool, R, nq, lens, cfg.scale, causal)
    for lay in (lambda t: t, apart, heads_first):
        lse = torch.full(q.shape[:2], float("nan"), device="cuda")
        out = lay(torch.full((sum(nq), H, R), float("nan"), dtype=DT[act], device="cuda"))
        run_cached(cfg, pool, lay(q), nq, lens, out, lse)
        check(out, lse, want, act)


@pytest.mark.parametrize("act,H,B,most", [("bf16", 16, 600, 90), ("bf16", 128, 40, 700), ("f32", 4, 600, 60), ("bf16", 8, 3, 20000)])
def test_cached_of_many_and_long_sequences(act, H, B, most):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, most, B)]
    nq = [int(x) for x in rng.integers(0, 3, B)]
    pool, q, cfg = cached_case(B, act, H, 512, 64, 32, nq, lens)
    out = run_cached(cfg, pool, q, nq, lens)
    check(out, None, ref.absorbed(q, pool, 512, nq, lens, cfg.scale), act)


def test_cached_same_results_each_time():
    nq, lens = [1, 2, 1], [3000, 700, 5]
    pool, q, cfg = cached_case(9, "bf16", 32, 512, 64, 64, nq, lens)
    first = run_cached(cfg, pool, q, nq, lens)
    for _ in range(5):
        assert torch.equal(run_cached(cfg, pool, q, nq, lens), first)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_cached_masks_pages_outside_the_pool(act):
    """Pages outside the pool are masked wherever they lie, up to a sequence of nothing else; lengths past the table
    are cut to it; rows that belong to no sequence stay."""
    page, nq, lens = 32, [1, 2, 1, 1], [300, 100, 64, 1000]
    pool, q, cfg = cached_case(4, act, 24, 512, 64, page, nq, [300, 100, 64, 320])
    pool.table[0, 0], pool.table[0, 3], pool.table[0, 9] = -1, pool.rows.shape[0], -2 ** 31
    pool.table[1, 1] = 2 ** 31 - 1
    pool.table[2, :2] = -1
    lse = torch.full((5, 24), float("nan"), device="cuda")
    out = run_cached(cfg, pool, q, nq, lens, lse=lse)
    want = ref.absorbed(q, pool, 512, nq, lens, cfg.scale)
    check(out, lse, want, act)
    assert (out[3] == 0).all() and torch.isneginf(lse[3]).all()
    extra = torch.full((9, 24, 512), 7.0, dtype=DT[act], device="cuda")
    more = torch.cat((q[:2], q, q[:2]))
    keep = (prefix(nq) + 2, i32(lens), i32(pool.table))
    gb.latent_cached(cfg, gb.attn_batch(*keep), more, gb.latent_cache(pool.rows), extra, workspace(cfg, 9, 4))
    # (more rows in the call: its work may be divided otherwise, so its sums may differ in their last bits)
    check(extra[2:7], None, want, act)
    assert (extra[:2] == 7.0).all() and (extra[7:] == 7.0).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 200, 298])
def test_cached_latents_that_are_no_numbers(act, bad, at):
    """They reach the queries that see them (their element at least), and no others: not the earlier draft tokens,
    not another sequence."""
    nq, lens = [4, 2], [300, 77]
    pool, q, cfg = cached_case(6, act, 20, 512, 64, 64, nq, lens)
    want = ref.absorbed(q, pool, 512, nq, lens, cfg.scale)
    pool.rows[pool.table[0, at // 64], at % 64, 17] = bad
    out = run_cached(cfg, pool, q, nq, lens)
    sees = [at <= 296 + i for i in range(4)] + [False, False]
    clean = torch.tensor(sees, device="cuda")
    assert not torch.isfinite(out[clean][..., 17]).any()
    whole = tuple(w[~clean] for w in want)
    check(out[~clean], None, whole, act)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_cached_queries_that_are_no_numbers(act):
    """A head of a token stays by itself."""
    nq, lens = [2], [500]
    pool, q, cfg = cached_case(8, act, 16, 512, 64, 64, nq, lens)
    want = ref.absorbed(q, pool, 512, nq, lens, cfg.scale)
    q[1, 3, 40] = float("nan")
    out = run_cached(cfg, pool, q, nq, lens)
    assert torch.isnan(out[1, 3]).all()
    keep = torch.ones((2, 16), dtype=torch.bool, device="cuda")
    keep[1, 3] = False
    check(out[keep][:, None], None, tuple(w[keep][:, None] if w.dim() == 3 else w[keep] for w in want), act)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_cached_scores_far_apart(act):
    """One key's score far above all others, wherever it lies (the maximum rises late), scores of thousands, and a
    query of zeros (all weights alike)."""
    lens = [700]
    for at in (0, 130, 699):
        pool, q, cfg = cached_case(10, act, 4, 512, 64, 64, [1], lens)
        pool.rows[pool.table[0, at // 64], at % 64] *= 8.0
        rows, _ = pool.sequence(0, 700)
        q[0, 0] = rows[at] * 4.0
        q[0, 1] = -rows[at] * 4.0
        q[0, 2] = 0.0
        out = run_cached(cfg, pool, q, [1], lens)
        # scores up to some 10^4: fp32 sums are off by about 2^-24 of it times a few, which the weights feel as it is
        check(out, None, ref.absorbed(q, pool, 512, [1], lens, cfg.scale), act, terms=2e-2)


@pytest.mark.parametrize("H", [3, 16, 30, 64, 128])
@pytest.mark.parametrize("R,P", [(512, 64), (128, 16)])
def test_cached_maxima_that_rise_in_every_tile(H, R, P):
    """Keys that grow along the sequence, so that the running maximum rises by far more than the weights are let run ahead
    in one tile after the other; 40 times, for tiles whose parts meet in any order."""
    lens, nq = [4000, 1100], [1, 1]
    pool, q, cfg = cached_case(12, "bf16", H, R, P, 64, nq, lens)
    for b, m in enumerate(lens):
        p = np.arange(m)
        rows = (torch.from_numpy(pool.table[b, p // 64]).long().cuda(), torch.from_numpy(p % 64).cuda())
        pool.rows[rows] = (pool.rows[rows].float() * torch.linspace(0.5, 12.0, m, device="cuda")[:, None]).to(torch.bfloat16)
    q[:, ::2] *= 4.0
    want = ref.absorbed(q, pool, R, nq, lens, cfg.scale)
    ws = workspace(cfg, 2, 2)
    outs = [run_cached(cfg, pool, q, nq, lens, ws=ws) for _ in range(40)]
    # scores up to some 10^3, whose fp32 sums are off by about 2^-24 of the sum of their products' sizes (several times
    # the score): up to 10^-3 of a weight
    check(outs[0], None, want, "bf16", terms=2e-3)
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("H,page", [(16, 16), (128, 64)])
def test_cached_waits_that_run_out(monkeypatch, H, page):
    nq, lens = [1, 2], [3000, 500]
    pool, q, cfg = cached_case(14, "bf16", H, 512, 64, page, nq, lens)
    keep, ws = (prefix(nq), i32(lens), i32(pool.table)), workspace(cfg, 3, 2)
    out = torch.zeros((3, H, 512), dtype=torch.bfloat16, device="cuda")
    monkeypatch.setenv("GBMOE_TC_WAIT_LIMIT_NS", "0")
    gb.latent_cached(cfg, gb.attn_batch(*keep), q, gb.latent_cache(pool.rows), out, ws)
    assert gb.moe_device_status(ws) == gb.EDEVICE_TIMEOUT
    monkeypatch.delenv("GBMOE_TC_WAIT_LIMIT_NS")
    check(run_cached(cfg, pool, q, nq, lens, ws=ws), None, ref.absorbed(q, pool, 512, nq, lens, cfg.scale), "bf16")


def test_cached_after_other_kernels():
    """Contexts of one to four tiles, each call after kernels of other code and sizes, so that the CTA's warps come to
    their first instructions at different times."""
    cases = [cached_case(20 + i, "bf16", H, R, P, page, [1] * len(lens), lens)
             for i, (H, R, P, page, lens) in enumerate([(1, 512, 64, 32, [127, 128]), (5, 256, 32, 16, [200, 17, 130]), (64, 512, 64, 64, [128]),
                                                        (30, 128, 16, 64, [250, 129, 64]), (128, 384, 64, 128, [190, 128])])]
    wants = [ref.absorbed(q, pool, cfg.latent_dim, [1] * q.shape[0], pool.lens, cfg.scale) for pool, q, cfg in cases]
    big = torch.empty(1 << 26, device="cuda")
    q, k, kr, v = prompt_inputs(1, "bf16", 8, 128, 64, 128, [300], [300])
    pc, o = gb.latent_config(8), torch.empty((300, 8, 128), dtype=torch.bfloat16, device="cuda")
    pws = workspace(pc, 300, 1)
    for _ in range(12):
        for (pool, cq, cfg), want in zip(cases, wants):
            big.fill_(1.0)
            gb.latent_prompt(pc, q, k, kr, v, prefix([300]), prefix([300]), o, pws)
            (big[: 1 << 20].view(1024, 1024) @ big[: 1 << 20].view(1024, 1024)).sum()
            check(run_cached(cfg, pool, cq, [1] * cq.shape[0], pool.lens), None, want, "bf16")


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_pool_past_32_bit_offsets(act):
    """A sequence's pages at the end of a pool of more than 2^32 bytes (and elements, bf16)."""
    page, W = 128, 576
    n = (1 << 32) // (page * W) + 40
    rows = torch.zeros((n, page, W), dtype=DT[act], device="cuda")
    pool = Pool.__new__(Pool)
    pool.page, pool.rows, pool.lens = page, rows, [300]
    pool.table = np.array([[n - 1, 3, n - 2]], dtype=np.int32)
    rows[pool.table[0].tolist()] = normal(2, (3, page, W), act)
    q = normal(1, (1, 16, W), act)
    cfg = gb.latent_config(16, act=act, page=page)
    out = run_cached(cfg, pool, q, [1], [300])
    check(out, None, ref.absorbed(q, pool, 512, [1], [300], cfg.scale), act)
    kv = normal(3, (1, W), act)
    keep = (prefix([1]), i32([301]), i32(pool.table))
    out = torch.empty_like(kv)
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, None, gb.attn_rope_table(64), gb.latent_cache(rows), kv_out=out)
    assert torch.equal(rows[n - 2, 300 - 256], out[0])


# ------------------------------------------------------------------- together


def test_both_forms_agree_and_run_on_another_stream():
    """A prompt in the expanded form, its last tokens again in the absorbed form over the cache that the append
    filled: keys W_k c and values W_v c, the same attention. On a stream of its own, and replayed from a graph."""
    H, R, P, N, V, lens, tail = 16, 512, 64, 128, 128, [200, 70], 2
    T = sum(lens)
    cfg = gb.latent_config(H, act="f32", page=32)
    wk, wv = normal(1, (H, N, R), "f32", R ** -0.5), normal(2, (H, V, R), "f32", R ** -0.5)
    kv, gamma, q = normal(3, (T, R + P), "f32", 2.0), normal(4, (R,), "f32").abs(), normal(5, (T, H, N + P), "f32")
    pool = Pool(0, "f32", R + P, 32, lens)
    table = gb.attn_rope_table(P)
    keep = (prefix(lens), i32(lens), i32(pool.table))
    ws = workspace(cfg, T, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    last = torch.cat([torch.arange(m - tail, m) + sum(lens[:b]) for b, m in enumerate(lens)]).cuda()
    few = (prefix([tail] * 2), i32(lens), keep[2])
    qa = torch.empty((2 * tail, H, R + P), device="cuda")
    lat = torch.empty((2 * tail, H, R), device="cuda")
    with torch.cuda.stream(side):
        gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, table, gb.latent_cache(pool.rows), q=q[..., N:], q_out=q[..., N:], kv_out=kv)
        k, v = torch.einsum("tr,hnr->thn", kv[:, :R], wk), torch.einsum("tr,hvr->thv", kv[:, :R], wv)
        out = torch.empty((T, H, V), device="cuda")
        gb.latent_prompt(cfg, q, k, kv[:, R:], v, keep[0], keep[0], out, ws)
        qa[..., :R], qa[..., R:] = torch.einsum("thn,hnr->thr", q[last, :, :N], wk), q[last, :, N:]
        gb.latent_cached(cfg, gb.attn_batch(*few), qa, gb.latent_cache(pool.rows), lat, ws)
        got = torch.einsum("thr,hvr->thv", lat, wv)
    side.synchronize()
    # products in fp32 (512 terms, TF32 off): either form is off by some 2^-24 of sums of about 1, and of the scores
    assert (got - out[last]).abs().max() <= 2e-4 * out.abs().max()
    graph, again = torch.cuda.CUDAGraph(), torch.zeros_like(lat)
    bundle, cache = gb.attn_batch(*few), gb.latent_cache(pool.rows)
    with torch.cuda.graph(graph):
        gb.latent_cached(cfg, bundle, qa, cache, again, ws)
    qa.mul_(0.5)  # the graph reads what is there when it runs
    graph.replay()
    gb.latent_cached(cfg, bundle, qa, cache, lat, ws)
    assert torch.equal(again, lat)
    assert gb.moe_device_status(ws) == gb.OK
