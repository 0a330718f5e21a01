"""Calls of latent attention that its header allows: padded batches, offsets past the batch, strides of 0, scales of
any sign, pages that several sequences have, many heads, streams beside each other, graphs that share a workspace."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2607_12875_gb300 as gb
from latent_reference import DT, Pool, check, i32, normal, prefix

pytestmark = pytest.mark.gpu


def workspace(cfg, T, B):
    return torch.zeros(gb.latent_workspace_size(cfg, T, B), dtype=torch.uint8, device="cuda")


def cached_case(seed, act, H, R, P, page, nq, lens, **kw):
    pool = Pool(seed, act, R + P, page, lens)
    return pool, normal(seed + 5, (sum(nq), H, R + P), act), gb.latent_config(H, latent_dim=R, rope_dim=P, act=act, page=page, **kw)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("nq,lens", [([1, 2], [300, 70]), ([3, 0], [0, 5]), ([4], [2])])
def test_rows_behind_the_last_sequence_are_left_as_they_were(act, nq, lens):
    """Nine tokens more than the sequences have; a last offset past the batch; lengths below 0 and past the table."""
    T, H = sum(nq), 6
    pool, q, cfg = cached_case(3, act, H, 256, 32, 32, nq, lens)
    q = torch.cat((q, torch.full_like(q[:1], float("nan")).expand(9, -1, -1)))
    out = torch.full((T + 9, H, 256), 7.0, dtype=DT[act], device="cuda")
    lse = torch.full((T + 9, H), 7.0, device="cuda")
    ws = workspace(cfg, T + 9, len(nq))
    gb.latent_cached(cfg, gb.attn_batch(prefix(nq), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
    check(out[:T], lse[:T], ref.absorbed(q[:T], pool, 256, nq, lens, cfg.scale), act)
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
    # the whole batch is the last sequence's, however far its offset lies; a length that is negative is none
    far = prefix(nq)
    far[-1] = 2 ** 31 - 1
    gb.latent_cached(cfg, gb.attn_batch(far, i32([*lens[:-1], -5]), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
    assert bool((out[sum(nq[:-1]):] == 0).all()) and bool(torch.isneginf(lse[sum(nq[:-1]):]).all())
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_prompt_rows_behind_the_last_sequence_are_left_as_they_were(act):
    nq, H = [140, 0, 5], 3
    T = sum(nq)
    cfg = gb.latent_config(H, act=act)
    q, k, kr, v = (normal(i, s, act) for i, s in enumerate([(T + 3, H, 192), (T + 3, H, 128), (T + 3, 64), (T + 3, H, 128)]))
    out, lse = torch.full((T + 3, H, 128), 7.0, dtype=DT[act], device="cuda"), torch.full((T + 3, H), 7.0, device="cuda")
    ws = workspace(cfg, T + 3, 3)
    gb.latent_prompt(cfg, q, k, kr, v, prefix(nq), prefix(nq), out, ws, lse=lse)
    check(out[:T], lse[:T], ref.expanded(q[:T], k[:T], kr[:T], v[:T], nq, nq, cfg.scale), act)
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_inputs_that_repeat_a_row(act):
    """Strides of 0: the same key for every head, the same rotary key and the same value for every token."""
    nq, H = [150, 20], 4
    T = sum(nq)
    cfg = gb.latent_config(H, act=act, causal=False)
    q, k = normal(1, (T, H, 192), act), normal(2, (T, 1, 128), act).expand(-1, H, -1)
    kr, v = normal(3, (1, 64), act).expand(T, -1), normal(4, (1, H, 128), act).expand(T, -1, -1)
    assert k.stride(1) == 0 and kr.stride(0) == 0 and v.stride(0) == 0
    for key, rope, value in [(k, kr, v), (k, kr.contiguous(), v.contiguous()), (k.contiguous(), kr, v.contiguous())]:
        out, ws = torch.full((T, H, 128), float("nan"), dtype=DT[act], device="cuda"), workspace(cfg, T, 2)
        gb.latent_prompt(cfg, q, key, rope, value, prefix(nq), prefix(nq), out, ws)
        check(out, None, ref.expanded(q, k, kr, v, nq, nq, cfg.scale, False), act)
    lens = [90, 200]
    pool, qc, cfg = cached_case(5, act, 8, 128, 64, 16, [1, 1], lens)
    qc = qc[:1, :1].expand(2, 8, -1)
    out, ws = torch.full((2, 8, 128), float("nan"), dtype=DT[act], device="cuda"), workspace(cfg, 2, 2)
    gb.latent_cached(cfg, gb.attn_batch(prefix([1, 1]), i32(lens), i32(pool.table)), qc, gb.latent_cache(pool.rows), out, ws)
    check(out, None, ref.absorbed(qc, pool, 128, [1, 1], lens, cfg.scale), act)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.05, 0.0, 1e-4, 0.25])
def test_scales_of_any_sign(act, scale):
    nq, H = [200, 31], 2
    cfg = gb.latent_config(H, act=act, scale=scale)
    T = sum(nq)
    q, k, kr, v = (normal(i + 9, s, act) for i, s in enumerate([(T, H, 192), (T, H, 128), (T, 64), (T, H, 128)]))
    out, lse = torch.full((T, H, 128), float("nan"), dtype=DT[act], device="cuda"), torch.empty((T, H), device="cuda")
    ws = workspace(cfg, T, 2)
    gb.latent_prompt(cfg, q, k, kr, v, prefix(nq), prefix(nq), out, ws, lse=lse)
    check(out, lse, ref.expanded(q, k, kr, v, nq, nq, cfg.scale), act)
    lens = [1000, 17]
    pool, q, cfg = cached_case(7, act, 20, 512, 64, 64, [1, 3], lens, scale=scale)
    out, lse = torch.full((4, 20, 512), float("nan"), dtype=DT[act], device="cuda"), torch.empty((4, 20), device="cuda")
    gb.latent_cached(cfg, gb.attn_batch(prefix([1, 3]), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
    check(out, lse, ref.absorbed(q, pool, 512, [1, 3], lens, cfg.scale), act)
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_sequences_that_share_pages(act):
    """A common beginning in the same pages, and one sequence with the same page twice."""
    lens, nq = [200, 180, 128], [1, 2, 1]
    pool, q, cfg = cached_case(11, act, 16, 512, 64, 32, nq, lens)
    pool.table[1, :4] = pool.table[0, :4]
    pool.table[2, 1:4] = pool.table[2, 0]
    pool.rows = torch.nan_to_num(pool.rows, 1.0)
    out, ws = torch.full((4, 16, 512), float("nan"), dtype=DT[act], device="cuda"), workspace(cfg, 4, 3)
    gb.latent_cached(cfg, gb.attn_batch(prefix(nq), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws)
    check(out, None, ref.absorbed(q, pool, 512, nq, lens, cfg.scale), act)


@pytest.mark.parametrize("act,H,R,P", [("bf16", 1000, 512, 64), ("bf16", 4096, 128, 16), ("f32", 600, 512, 128), ("bf16", 513, 512, 128)])
def test_many_heads(act, H, R, P):
    """More rows than the CTAs beside each other take, with a share's end inside a sequence's."""
    lens, nq = [700, 64], [2, 1]
    pool, q, cfg = cached_case(13, act, H, R, P, 64, nq, lens)
    out, lse = torch.full((3, H, R), float("nan"), dtype=DT[act], device="cuda"), torch.empty((3, H), device="cuda")
    ws = workspace(cfg, 3, 2)
    gb.latent_cached(cfg, gb.attn_batch(prefix(nq), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
    check(out, lse, ref.absorbed(q, pool, R, nq, lens, cfg.scale), act)
    assert gb.moe_device_status(ws) == gb.OK


def test_calls_beside_each_other():
    """Two streams with a workspace each, calls of both forms in flight at the same time."""
    H, nq, lens = 32, [1] * 6, [2000, 90, 5000, 1, 700, 64]
    pool, q, cfg = cached_case(17, "bf16", H, 512, 64, 64, nq, lens)
    n = [700, 300]
    pq, k, kr, v = (normal(i + 20, s, "bf16") for i, s in enumerate([(1000, H, 192), (1000, H, 128), (1000, 64), (1000, H, 128)]))
    want_c = ref.absorbed(q, pool, 512, nq, lens, cfg.scale)
    want_p = ref.expanded(pq, k, kr, v, n, n, cfg.scale)
    keep = (prefix(nq), i32(lens), i32(pool.table))
    cu = prefix(n)
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    torch.cuda.synchronize()
    for turn in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                ws = workspace(cfg, 1000, 6)
                if (turn + i) % 2:
                    out = torch.full((6, H, 512), float("nan"), dtype=torch.bfloat16, device="cuda")
                    gb.latent_cached(cfg, gb.attn_batch(*keep), q, gb.latent_cache(pool.rows), out, ws)
                else:
                    out = torch.full((1000, H, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
                    gb.latent_prompt(cfg, pq, k, kr, v, cu, cu, out, ws)
                outs.append((out, ws, (turn + i) % 2))
    torch.cuda.synchronize()
    for out, ws, c in outs:
        check(out, None, want_c if c else want_p, "bf16")
        assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_graphs_of_a_step_share_a_workspace(act):
    """Norm, append and attention of single tokens captured twice (other inputs) with one workspace between them and
    replayed in turn: lengths and offsets are what the device holds then, whatever they were at the capture."""
    H, R, P, page, B = 16, 512, 64, 16, 3
    W, Hd = R + P, 1024
    cfg = gb.latent_config(H, act=act, page=page)
    layer = gb.make_config(B, Hd, 128, 8, 2, act=act, w=act)
    lens = [40, 1, 333]
    pool = Pool(19, act, W, page, [n + 40 for n in lens], poison=False)
    cache, table = gb.latent_cache(pool.rows), gb.attn_rope_table(P)
    kv_len = i32(lens)
    keep = (prefix([1] * B), kv_len, i32(pool.table))
    batch = gb.attn_batch(*keep)
    ws = workspace(cfg, B, B)
    steps = []
    for g in range(2):
        t = dict(x=normal(g, (B, Hd), act), r=normal(g + 30, (B, Hd), act), y=torch.empty((B, Hd), dtype=DT[act], device="cuda"),
                 gamma=normal(g + 40, (Hd,), act), kv=normal(g + 50, (B, W), act), q=normal(g + 60, (B, H, W), act),
                 out=torch.empty((B, H, R), dtype=DT[act], device="cuda"))
        qt = torch.empty_like(t["q"])

        def step(t=t, qt=qt):
            gb.moe_rmsnorm_add(layer, t["x"], t["r"], t["gamma"], 1e-6, None, t["y"])
            qt.copy_(t["q"])
            gb.latent_append(cfg, batch, t["kv"], None, table, cache, q=t["q"][..., R:], q_out=qt[..., R:])
            gb.latent_cached(cfg, batch, qt, cache, t["out"], ws)
        step()  # (outside of a capture first: what is set up once)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        steps.append((graph, t, qt))
    now = list(lens)
    for i in range(6):
        graph, t, qt = steps[i % 2]
        now = [n + 3 for n in now]
        kv_len.copy_(i32(now))
        t["kv"].copy_(normal(100 + i, (B, W), act))
        t["out"].fill_(float("nan"))
        graph.replay()
        check(t["out"], None, ref.absorbed(qt, pool, R, [1] * B, now, cfg.scale), act)
        for b, n in enumerate(now):  # the row that was appended (its latent as it is: no gamma)
            assert torch.equal(pool.rows[pool.table[b, (n - 1) // page], (n - 1) % page, :R], t["kv"][b, :R])
        plain = torch.empty_like(t["y"])
        gb.moe_rmsnorm(layer, t["x"] + t["r"], t["gamma"], 1e-6, plain)
        assert torch.equal(plain, t["y"])
    assert gb.moe_device_status(ws) == gb.OK


def test_append_of_padded_and_clamped_batches():
    """Tokens behind the last sequence have no place and no outputs; explicit positions may be anything."""
    R, P, page, H = 64, 32, 16, 3
    cfg = gb.latent_config(H, latent_dim=R, rope_dim=P, act="f32", page=page, rotary_layout="half")
    pool = torch.full((4, page, R + P), 7.0, device="cuda")
    kv, q = normal(1, (9, R + P), "f32"), normal(2, (9, H, P), "f32")
    kv_out, q_out = torch.full((9, R + P), 7.0, device="cuda"), torch.full((9, H, P), 7.0, device="cuda")
    pos = i32([-3, 2 ** 31 - 1, 0, 5, 5, 5, 5, 5, 5])
    cu, lens, ids, table = prefix([2, 3]), i32([17, 18]), i32([[2, 0], [1, -1]]), gb.attn_rope_table(P)
    gb.latent_append(cfg, gb.attn_batch(cu, lens, ids), kv, None, table, gb.latent_cache(pool), q=q, q_out=q_out, kv_out=kv_out,
                     positions=pos)
    assert torch.equal(kv_out[:5, :R], kv[:5, :R])
    assert bool((kv_out[5:] == 7).all()) and bool((q_out[5:] == 7).all())
    stored = torch.zeros((4, page), dtype=torch.bool, device="cuda")
    for page_id, slot, t in [(2, 15, 0), (0, 0, 1), (1, 15, 2)]:  # (the second sequence's last two: no such page)
        stored[page_id, slot] = True
        assert torch.equal(pool[page_id, slot], kv_out[t])
    assert bool((pool[~stored] == 7).all())
    # rotations keep a pair's length, whatever the position
    a, b = q[:5].double(), q_out[:5].double()
    assert torch.allclose(a[..., :16] ** 2 + a[..., 16:] ** 2, b[..., :16] ** 2 + b[..., 16:] ** 2, rtol=1e-5, atol=1e-6)
    # an offset past the batch: the last sequence has all of the rest
    pool.fill_(7.0)
    cu[-1], lens[1] = 1000, 12
    gb.latent_append(cfg, gb.attn_batch(cu, lens, ids), kv, None, table, gb.latent_cache(pool), kv_out=kv_out)
    assert torch.equal(pool[1, 5:12], kv_out[2:]) and bool((pool[1, :5] == 7).all()) and bool((pool[1, 12:] == 7).all())


def test_sizes_at_the_limits():
    """One token and one key; R of 512 with P of 128; heads past a warp's; a batch of empty sequences only."""
    for act in ("f32", "bf16"):
        for R, P in [(8, 0), (8, 16), (512, 128), (512, 64), (128, 0)]:
            pool, q, cfg = cached_case(23, act, 1, R, P, 16, [1], [1])
            out, ws = torch.full((1, 1, R), float("nan"), dtype=DT[act], device="cuda"), workspace(cfg, 1, 1)
            gb.latent_cached(cfg, gb.attn_batch(prefix([1]), i32([1]), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws)
            check(out, None, ref.absorbed(q, pool, R, [1], [1], cfg.scale), act)
            keep = prefix([0] * 40), i32(np.zeros(40)), i32(np.zeros((40, 1)))
            out.fill_(7.0)
            gb.latent_cached(cfg, gb.attn_batch(*keep), q, gb.latent_cache(pool.rows), out, ws)
            assert bool((out == 7).all()) and gb.moe_device_status(ws) == gb.OK
        for N, P, V in [(8, 0, 8), (8, 16, 8), (128, 128, 128), (128, 64, 128), (72, 48, 104)]:
            cfg = gb.latent_config(1, rope_dim=P, nope_dim=N, value_dim=V, act=act)
            q, k, v = normal(1, (1, 1, N + P), act), normal(2, (1, 1, N), act), normal(3, (1, 1, V), act)
            kr = normal(4, (1, P), act) if P else None
            out, ws = torch.full((1, 1, V), float("nan"), dtype=DT[act], device="cuda"), workspace(cfg, 1, 1)
            gb.latent_prompt(cfg, q, k, kr, v, prefix([1]), prefix([1]), out, ws)
            assert torch.equal(out, v)  # (one key: its weight is 1)
            out.fill_(7.0)
            gb.latent_prompt(cfg, q, k, kr, v, prefix([0, 0]), prefix([1, 0]), out, ws)
            assert bool((out == 7).all()) and gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("H,nq,lens", [
    (64, [200], [600]),                                   # more tiles of rows than shares
    (16, [1] * 32, [900] * 31 + [64]), (16, [1] * 33, [900] * 32 + [64]),  # sequences that a warp looks through, and one more
    (40, [1] * 5, [9000, 1, 0, 64, 65]),                  # one of them nearly all of the work
    (24, [0, 3, 0, 1, 0], [500, 2000, 0, 1999, 7]),       # sequences without queries in between
    (128, [1] * 3, [6400, 6464, 6336]),
])
def test_shares_of_the_key_axis(H, nq, lens):
    """Parts of tiles, shares over several tiles, idle ones: every key is seen once."""
    pool, q, cfg = cached_case(29, "bf16", H, 512, 64, 64, nq, lens)
    out, lse = torch.full((sum(nq), H, 512), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.empty((sum(nq), H), device="cuda")
    ws = workspace(cfg, sum(nq), len(nq))
    for _ in range(2):
        gb.latent_cached(cfg, gb.attn_batch(prefix(nq), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws, lse=lse)
        check(out, lse, ref.absorbed(q, pool, 512, nq, lens, cfg.scale), "bf16")
    assert gb.moe_device_status(ws) == gb.OK


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("page,R,P,H,new,lens", [
    (16, 512, 64, 5, [1, 1, 1], [1, 17, 32]), (64, 512, 64, 128, [70, 0, 3], [200, 64, 3]), (128, 8, 128, 3, [300, 5], [300, 131]),
    (32, 256, 32, 16, [1] * 70, list(range(1, 71))),
])
@pytest.mark.parametrize("queries,rows_out", [(False, False), (True, False), (False, True)])
def test_append_stores_the_same_rows_whatever_else_is_wanted(act, page, R, P, H, new, lens, queries, rows_out):
    """The rows that a call with every output gives (held to 64 bits elsewhere) in their slots bit for bit, and every other
    slot as it was, with none or one of the optional outputs."""
    T = sum(new)
    pool = Pool(page, act, R + P, page, lens)
    kv, gamma, q = normal(1, (T, R + P), act, 3.0), normal(2, (R,), act), normal(3, (T, H, P), act)
    cfg, table = gb.latent_config(H, latent_dim=R, rope_dim=P, act=act, page=page), gb.attn_rope_table(P)
    keep = (prefix(new), i32(lens), i32(pool.table))
    want_kv, want_q = torch.empty_like(kv), torch.empty_like(q)
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, table, gb.latent_cache(pool.rows.clone()), q=q, q_out=want_q, kv_out=want_kv)
    want, at = pool.rows.clone(), 0
    for b, (n, m) in enumerate(zip(new, lens)):
        for p in range(m - n, m):
            want[pool.table[b, p // page], p % page] = want_kv[at]
            at += 1
    got_kv, got_q = torch.full_like(kv, 7.0), torch.full_like(q, 7.0)
    outputs = {**(dict(q=q, q_out=got_q) if queries else {}), **(dict(kv_out=got_kv) if rows_out else {})}
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, gamma, table, gb.latent_cache(pool.rows), **outputs)
    bits = torch.int32 if act == "f32" else torch.int16
    assert torch.equal(pool.rows.view(bits), want.view(bits))
    assert torch.equal(got_q, want_q) if queries else bool((got_q == 7).all())
    assert torch.equal(got_kv, want_kv) if rows_out else bool((got_kv == 7).all())


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
@pytest.mark.parametrize("shared", [True, False])
def test_prompt_keys_with_an_infinity(act, bad, shared):
    """One element of a key (of its rotary part, all heads', or of one head's own): for a query that sees it the score is
    +inf or -inf by the sign of the query's element, so its result is no number, or the one without that key."""
    lens, H, N, at = [100, 37, 129], 3, 128, 120                # position 20 of the second sequence
    T = sum(lens)
    q, k, kr, v = (normal(i + 31, s, act) for i, s in enumerate([(T, H, 192), (T, H, N), (T, 64), (T, H, 128)]))
    cfg = gb.latent_config(H, act=act)
    want = ref.expanded(q, k, kr, v, lens, lens, cfg.scale)
    two = slice(100, 137)
    present = torch.ones(37, dtype=torch.bool, device="cuda")
    present[at - 100] = False
    key = torch.cat((k, kr[:, None].expand(-1, H, -1)), -1)
    without = ref.attention(q[two], key[two], v[two], 37, 37, cfg.scale, True, present)
    if shared:
        kr[at, 5] = bad
        score = bad * q[two, :, N + 5].double()
    else:
        k[at, 1, 7] = bad
        score = torch.zeros((37, H), dtype=torch.float64, device="cuda")
        score[:, 1] = bad * q[two, 1, 7].double()
    sees = torch.arange(37, device="cuda")[:, None] >= at - 100
    up, down = sees & (score == torch.inf), sees & (score == -torch.inf)
    assert bool(up.any()) and bool(down.any())
    out, ws = torch.full((T, H, 128), 7.0, dtype=DT[act], device="cuda"), workspace(cfg, T, 3)
    gb.latent_prompt(cfg, q, k, kr, v, prefix(lens), prefix(lens), out, ws)
    assert gb.moe_device_status(ws) == gb.OK
    mine = out[two]
    assert bool(torch.isnan(mine[up]).all())
    check(mine[down][:, None], None, tuple(w[down][:, None] if w.dim() == 3 else w[down] for w in without), act)
    rest = torch.ones((T, H), dtype=torch.bool, device="cuda")
    rest[two] = ~(up | down)
    check(out[rest][:, None], None, tuple(w[rest][:, None] if w.dim() == 3 else w[rest] for w in want), act)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 200, 298])
def test_cached_rotary_keys_with_an_infinity(act, bad, at):
    """The same over cached rows: draft tokens of which some do not see the row, and a sequence without it."""
    nq, lens, H, R = [4, 2], [300, 77], 20, 512
    pool, q, cfg = cached_case(17, act, H, R, 64, 64, nq, lens)
    want = ref.absorbed(q, pool, R, nq, lens, cfg.scale)
    rows, _ = pool.sequence(0, 300)
    key = rows[:, None].expand(-1, H, -1)
    present = torch.arange(300, device="cuda") != at
    without = ref.attention(q[:4], key, key[..., :R], 4, 300, cfg.scale, True, present)
    pool.rows[pool.table[0, at // 64], at % 64, R + 5] = bad
    sees = (torch.arange(296, 300, device="cuda") >= at)[:, None]
    score = bad * q[:4, :, R + 5].double()
    up, down = sees & (score == torch.inf), sees & (score == -torch.inf)
    assert bool(up.any()) and bool(down.any())
    out, ws = torch.full((6, H, R), 7.0, dtype=DT[act], device="cuda"), workspace(cfg, 6, 2)
    gb.latent_cached(cfg, gb.attn_batch(prefix(nq), i32(lens), i32(pool.table)), q, gb.latent_cache(pool.rows), out, ws)
    assert gb.moe_device_status(ws) == gb.OK
    assert bool(torch.isnan(out[:4][up]).all())
    check(out[:4][down][:, None], None, tuple(w[down][:, None] if w.dim() == 3 else w[down] for w in without), act)
    rest = torch.ones((6, H), dtype=torch.bool, device="cuda")
    rest[:4] = ~(up | down)
    check(out[rest][:, None], None, tuple(w[rest][:, None] if w.dim() == 3 else w[rest] for w in want), act)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("B", [256, 257, 1100])
def test_append_of_many_sequences(act, B):
    """More sequences than are looked through at once, most of them with no or one token: each token's row in its own slot,
    the values of a call without norm (the latent as it is), every other slot and row as it was."""
    rng = np.random.default_rng(B)
    new = [int(n) for n in rng.choice([0, 0, 1, 1, 2, 7], B)]
    lens = [n + int(m) for n, m in zip(new, rng.integers(0, 40, B))]
    R, P, page, T = 64, 16, 16, sum(new)
    pool = Pool(31, act, R + P, page, lens)
    kv, q = normal(1, (T + 5, R + P), act), normal(2, (T + 5, 2, P), act)
    cfg, table = gb.latent_config(2, latent_dim=R, rope_dim=P, act=act, page=page), gb.attn_rope_table(P)
    kv_out, q_out = torch.full_like(kv, 7.0), torch.full_like(q, 7.0)
    want = pool.rows.clone()
    keep = (prefix(new) + 2, i32(lens), i32(pool.table))
    gb.latent_append(cfg, gb.attn_batch(*keep), kv, None, table, gb.latent_cache(pool.rows), q=q, q_out=q_out, kv_out=kv_out)
    mine = slice(2, T + 2)
    at = np.concatenate([np.arange(m - n, m) for n, m in zip(new, lens)])
    seq = np.repeat(np.arange(B), new)
    want[torch.from_numpy(pool.table[seq, at // page]).long().cuda(), torch.from_numpy(at % page).cuda()] = kv_out[mine]
    bits = torch.int32 if act == "f32" else torch.int16
    assert torch.equal(pool.rows.view(bits), want.view(bits)) and torch.equal(kv_out[mine, :R], kv[mine, :R])
    # the turns are those of the tokens' places: one sequence with the same positions gives the same
    flat_kv, flat_q = torch.empty_like(kv[mine]), torch.empty_like(q[mine])
    one = torch.zeros((T // page + 1, page, R + P), dtype=DT[act], device="cuda")
    keep = (prefix([T]), i32([T]), i32([list(range(T // page + 1))]), i32(at))
    gb.latent_append(cfg, gb.attn_batch(*keep[:3]), kv[mine], None, table, gb.latent_cache(one), q=q[mine], q_out=flat_q, kv_out=flat_kv,
                     positions=keep[3])
    assert torch.equal(kv_out[mine], flat_kv) and torch.equal(q_out[mine], flat_q)
    for t in (kv_out, q_out):
        assert bool((t[:2] == 7).all()) and bool((t[T + 2:] == 7).all())
