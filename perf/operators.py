"""What the attention operators are measured on: the half of a decoder layer
that stands before the MoE layer, as a serving program runs it.

Four operators: rotary positions (rope), appending keys and values to a paged
cache with the rotation on the way (append), causal attention over packed
prompts (prompt), and attention of few query tokens per sequence over the
paged cache (cached). Head counts are the benchmark workloads' hidden sizes
over their head size (1024, 4096, 7168: 16 heads of 64, 32 and 56 of 128), the
token counts those of its decode and prefill batches; draw() spreads sizes,
types, layouts and lengths over the ranges between them.

With `own` false the operators run in their plain form, elementary torch
operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0


def _case(name, op, **kw):
    c = dict(op=op, heads=32, kv_heads=8, dim=128, act="bf16", rotary=0, layout="half", base=10000.0, factor=1.0)
    if op in ("append", "cached"):
        c.update(cache="e4m3", page=64)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode batch of 32 sequences: one token each, launch latency only
        _case("rope_decode_T32", "rope", T=32, ctx=32768, rotary=128),
        # a prefill batch with part of each head rotated, interleaved pairs, frequencies scaled for long contexts
        _case("rope_prompt_T8192", "rope", T=8192, ctx=131072, rotary=64, layout="interleaved", base=500000.0, factor=8.0),
        # one decoded token of each of 128 sequences goes to the 8-bit cache, queries rotated in the same pass
        _case("append_decode_e4m3_B128", "append", B=128, new=128, ctx=8192, rotary=128),
        # a prefill batch of packed prompts fills its pages
        _case("append_prompt_e4m3_T8192", "append", B=5, new=8192, ctx=8192, rotary=128, base=500000.0, factor=8.0),
        # a small model's odd batch into a cache of the activations' own type, small pages
        _case("append_bf16_T777", "append", B=3, new=777, ctx=1500, heads=16, kv_heads=16, dim=64, rotary=32,
              layout="interleaved", cache="act", page=16),
        # a full-precision run of a small model: three short prompts
        _case("prompt_f32_T333", "prompt", B=3, T=333, heads=16, kv_heads=4, dim=64, act="f32"),
        # packed prompts of very different lengths, together a prefill batch
        _case("prompt_packed_T8192", "prompt", B=7, T=8192),
        # one long prompt
        _case("prompt_long_T16384", "prompt", B=1, T=16384),
        # one sequence being decoded
        _case("cached_e4m3_B1", "cached", B=1, q_len=1, ctx=4000),
        # several draft tokens per sequence checked at once, small heads, cache in bf16, small pages
        _case("cached_bf16_B17_q4", "cached", B=17, q_len=4, ctx=3000, heads=16, kv_heads=4, dim=64, cache="act", page=16),
        # a decode batch of 32 sequences of up to 32768 tokens
        _case("cached_e4m3_B32", "cached", B=32, q_len=1, ctx=32768),
        # few very long contexts, seven query heads per cached head
        _case("cached_e4m3_B4_long", "cached", B=4, q_len=1, ctx=131072, heads=56),
    ]


def draw(rng):
    """One of the four operators with other sizes: token counts and lengths over
    their logarithm, head counts, head sizes, layouts and types as they come."""
    def log_int(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    op = rng.choice(["rope", "append", "prompt", "prompt", "cached", "cached"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8])
    kw = dict(dim=dim, kv_heads=kv, heads=kv * rng.choice([1, 2, 4, 6, 7, 8]))
    if op in ("rope", "append"):
        kw.update(rotary=rng.choice([dim // 4, dim // 2, dim, dim]), layout=rng.choice(["half", "interleaved"]),
                  base=rng.choice([10000.0, 500000.0]), factor=rng.choice([1.0, 4.0, 8.0]))
    f32 = rng.random() < 0.2
    kw["act"] = "f32" if f32 else "bf16"
    if op == "rope":
        return _case(None, op, T=log_int(1, 8192), ctx=log_int(9000, 131072), **kw)
    if op == "append":
        B = log_int(1, 128)
        new = 1 if rng.random() < 0.4 else log_int(2, max(2, 8192 // B))
        return _case(None, op, B=B, new=B if new == 1 else B * new + rng.randint(0, B - 1), ctx=log_int(new + 1, 16384),
                     cache=rng.choice(["act", "e4m3", "e4m3"]), page=rng.choice([16, 32, 64, 128]), **kw)
    if op == "prompt":
        T = log_int(16, 600 if f32 else 9000)
        return _case(None, op, B=log_int(1, min(16, T)), T=T, **kw)
    B = log_int(1, 64)
    most = (1 << 19) // B  # tokens in all
    return _case(None, op, B=B, q_len=rng.choice([1, 1, 1, 2, 5]), ctx=log_int(1, min(most, 4096 if f32 else 131072)),
                 cache=rng.choice(["act", "e4m3", "e4m3"]), page=rng.choice([16, 32, 64, 128]), **kw)


# ---------------------------------------------------------------- sizes of a case


def _parts(total, n, key):
    """total split into n uneven parts of at least 1 (when it reaches)."""
    r = random.Random(key)
    w = [r.uniform(0.2, 2.0) for _ in range(n)]
    spare = max(0, total - n)
    cut = [round(spare * sum(w[:i]) / sum(w)) for i in range(n + 1)]
    return [cut[i + 1] - cut[i] + (1 if i < total else 0) for i in range(n)]


def _shape(c):
    """New (query) tokens of each sequence and the keys each has after them."""
    if c["op"] == "rope":
        return [c["T"]], [c["ctx"]]
    if c["op"] == "prompt":
        lens = _parts(c["T"], c["B"], 77 * c["T"] + c["B"])
        return lens, lens
    B = c["B"]
    r = random.Random(31 * c["ctx"] + B)
    new = [c["q_len"]] * B if c["op"] == "cached" else _parts(c["new"], B, 13 * c["new"] + B)
    # lengths from an eighth of the longest on, one of them the longest
    lens = [c["ctx"] if i == 0 else r.randint(max(1, c["ctx"] // 8), c["ctx"]) for i in range(B)]
    if c["op"] == "append":  # every new token has a place
        lens = [max(n, m) for n, m in zip(new, lens)]
    return new, lens


def _freqs(c):
    """Angle per position of each pair (radians), and the factor of cos and sin:
    base^(-2i/R); with a factor, frequencies that turn less than once within the
    original 8192 positions are divided by it, those that turn over 32 times are
    kept, with a ramp between, and the factor is 0.1 ln(factor) + 1."""
    R = c["rotary"]
    f = [c["base"] ** (-2.0 * i / R) for i in range(R // 2)]
    if c["factor"] == 1.0:
        return f, 1.0

    def at(turns):
        return R * math.log(8192 / (turns * 2 * math.pi)) / (2 * math.log(c["base"]))
    lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), R - 1)
    out = []
    for i, v in enumerate(f):
        ramp = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
        out.append(v * (1.0 - ramp) + v / c["factor"] * ramp)
    return out, 0.1 * math.log(c["factor"]) + 1.0


# ---------------------------------------------------------------- inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dt, sigma=1.0):
    return torch.empty(shape, device=DEV).normal_(0.0, sigma, generator=g).to(dt)


def _keys(g, shape, dt):
    """Keys: some channels of each head larger than the others, as models have them."""
    gain = torch.empty(shape[1:], device=DEV).normal_(0.0, 0.4, generator=g).exp_()
    return (torch.empty(shape, device=DEV).normal_(0.0, 1.0, generator=g) * gain).to(dt)


def _prefix(v):
    return torch.tensor([sum(v[:i]) for i in range(len(v) + 1)], dtype=torch.int32, device=DEV)


def _pages(c, g, lens):
    """A page table over a pool in which every sequence's pages lie scattered."""
    per = max(1, max(-(-n // c["page"]) for n in lens))
    used = [-(-n // c["page"]) for n in lens]
    order = torch.randperm(sum(used) + 3, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((len(lens), per), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(used) + 3


def _pool(c, g, n_pages, keys):
    """Cached keys or values: codes and scale bytes, or values of the activations' type."""
    shape = (n_pages, c["kv_heads"], c["page"], c["dim"])
    dt = torch.float32 if c["act"] == "f32" else torch.bfloat16
    x = torch.empty(shape, device=DEV).normal_(0.0, 1.0, generator=g)
    if keys:
        x *= torch.empty((1, shape[1], 1, shape[3]), device=DEV).normal_(0.0, 0.4, generator=g).exp_()
    if c["cache"] == "act":
        return x.to(dt), None
    e = torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / E4M3_MAX))
    codes = (x * torch.exp2(-e)[:, :, None, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (e + 127.0).to(torch.uint8)


def _inputs(c, seed):
    g = _gen(seed)
    dt = torch.float32 if c["act"] == "f32" else torch.bfloat16
    new, lens = _shape(c)
    T, Hq, Hkv, D = sum(new), c["heads"], c["kv_heads"], c["dim"]
    d = {"case": c, "q": _normal(g, (T, Hq, D), dt, 1.5)}
    if c["op"] != "cached":  # keys and values as slices of one projection's rows
        kv = torch.empty((T, 2 * Hkv, D), dtype=dt, device=DEV)
        kv[:, :Hkv] = _keys(g, (T, Hkv, D), dt)
        kv[:, Hkv:] = _normal(g, (T, Hkv, D), dt)
        d["k"], d["v"] = kv[:, :Hkv], kv[:, Hkv:]
    d["cu"] = _prefix(new)
    d["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if c["op"] in ("append", "cached"):
        d["table"], n = _pages(c, g, lens)
        d["k_pool"], d["k_scale"] = _pool(c, g, n, True)
        d["v_pool"], d["v_scale"] = _pool(c, g, n, False)
    if c["op"] == "rope":
        d["pos"] = torch.randint(0, c["ctx"], (T,), generator=g, device=DEV, dtype=torch.int32)
        d["k_out"] = torch.empty((T, Hkv, D), dtype=dt, device=DEV)
    if c["rotary"]:
        f, d["mag"] = _freqs(c)
        d["freqs"] = torch.tensor(f, dtype=torch.float64, device=DEV)
        # turns per position as a 64-bit binary fraction: what the framework's rotations take
        turns = [int(v / (2 * math.pi) * 2.0 ** 64) % (1 << 64) for v in f]
        d["turns"] = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device=DEV)
    d["out"] = torch.empty_like(d["q"])
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    if own:  # the handles that a program keeps: config, pointer bundles, workspace
        import paper_2607_12875_gb300 as gb
        c = case
        d["gb"] = gb
        d["cfg"] = gb.attn_config(c["heads"], c["kv_heads"], c["dim"], act=c["act"], rotary_dim=c["rotary"],
                                  rotary_layout=c["layout"], rotary_scale=d.get("mag", 1.0), cache=c.get("cache", "act"),
                                  page=c.get("page", 64))
        if c["op"] in ("append", "cached"):
            d["batch"] = gb.attn_batch(d["cu"], d["lens"], d["table"])
            d["bundle"] = gb.attn_cache(d["k_pool"], d["v_pool"], d["k_scale"], d["v_scale"])
        d["ws"] = torch.empty(gb.attn_workspace_size(d["cfg"], d["q"].shape[0], d["lens"].numel()), dtype=torch.uint8,
                              device=DEV)
    return d


# ---------------------------------------------------------------- plain forms


def _rotate(c, x, pos, freqs, mag):
    """x [T, H, D] rotated, in 32 bits (angles in 64: positions times frequencies do not fit 32)."""
    R, x = c["rotary"], x.float()
    a = pos.double()[:, None] * freqs
    cos, sin = (a.cos() * mag).float()[:, None], (a.sin() * mag).float()[:, None]
    if c["layout"] == "half":
        u, w = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((u * cos - w * sin, u * sin + w * cos), -1)
    else:
        u, w = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((u * cos - w * sin, u * sin + w * cos), -1).flatten(-2)
    return torch.cat((y, x[..., R:]), -1)


def _new_positions(s):
    """Sequence and position of every new token."""
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=s["q"].shape[0])
    pos = torch.arange(s["q"].shape[0], device=DEV) - s["cu"][seq].long() + (s["lens"].long() - n)[seq]
    return seq, pos


def _store(c, pool, scale, x, page, off):
    """x [T, Hkv, D] to slot off of each token's page, in place; the page's scale covers old and new tokens."""
    if scale is None:
        pool[page, :, off] = x.to(pool.dtype)
        return
    touched, at = torch.unique_consecutive(page, return_inverse=True)  # the pages that get tokens
    shape = (touched.numel(), scale.shape[1])
    top = torch.zeros(shape, device=DEV).index_reduce_(0, at, x.abs().amax(-1), "amax")
    first = torch.full(shape[:1], c["page"], device=DEV).index_reduce_(0, at, off, "amin")  # tokens before the new ones
    need = torch.ceil(torch.log2(top / E4M3_MAX)).clamp(-127, 127)
    old = scale[touched].float() - 127.0
    e = torch.where((first == 0)[:, None], need, torch.maximum(old, need))
    keep = torch.arange(c["page"], device=DEV) < first[:, None]  # rescaled where tokens were before
    grow = torch.where(keep[:, None, :], torch.exp2(old - e)[:, :, None], 1.0)[..., None]
    codes = pool.view(torch.float8_e4m3fn)
    pool[touched] = (codes[touched].float() * grow).to(torch.float8_e4m3fn).view(torch.uint8)
    pool[page, :, off] = (x * torch.exp2(-e[at])[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    scale[touched] = (e + 127.0).to(torch.uint8)


def _weighted(s, see, v):
    """softmax over the keys seen (none: 0), times v."""
    s = s.masked_fill_(~see, -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    return (p @ v) / p.sum(-1, keepdim=True).clamp_min(1e-38)


def _plain_prompt(s):
    c = s["case"]
    G, D = c["heads"] // c["kv_heads"], c["dim"]
    outs, at = [], 0
    for n in _shape(c)[0]:  # a sequence at a time: together their score matrices would be mostly masked
        q = s["q"][at:at + n].float().view(n, -1, G, D).permute(1, 2, 0, 3)
        k, v = (s[w][at:at + n].float().transpose(0, 1)[:, None] for w in ("k", "v"))
        see = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        outs.append(_weighted((q * D ** -0.5) @ k.transpose(-1, -2), see, v).permute(2, 0, 1, 3).reshape(n, -1, D))
        at += n
    return torch.cat(outs).to(s["q"].dtype)


def _gather(c, pool, scale, table):
    """Every sequence's cached rows [B, Hkv, pages * page, D] in 32 bits."""
    x = (pool if scale is None else pool.view(torch.float8_e4m3fn))[table.long()].float()
    if scale is not None:
        x *= torch.exp2(scale[table.long()].float() - 127.0)[..., None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_cached(s):
    c = s["case"]
    B, n, Hkv, D = c["B"], c["q_len"], c["kv_heads"], c["dim"]
    G = c["heads"] // Hkv
    k, v = (_gather(c, s[w + "_pool"], s[w + "_scale"], s["table"]) for w in ("k", "v"))
    q = s["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    pos = s["lens"][:, None] - n + torch.arange(n, device=DEV)  # of each query token
    see = torch.arange(k.shape[2], device=DEV) <= pos.repeat_interleave(G, 1)[..., None]
    o = _weighted((q * D ** -0.5) @ k.transpose(-1, -2), see[:, None], v)
    return o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B * n, -1, D).to(s["q"].dtype)


# ---------------------------------------------------------------- a pass


def _cache_out(s, r):
    """The cache as it now is: codes and scales as the numbers they stand for."""
    for w in ("k", "v"):
        r[w + "_pool"] = s[w + "_pool"] if s[w + "_scale"] is None else s[w + "_pool"].view(torch.float8_e4m3fn)
        if s[w + "_scale"] is not None:
            r[w + "_scale"] = s[w + "_scale"].view(torch.float8_e8m0fnu)
    return r


def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        gb = s["gb"]
        if op == "rope":
            gb.attn_rope(s["cfg"], s["q"], s["k"], s["pos"], s["turns"], s["out"], s["k_out"])
            return {"q": s["out"], "k": s["k_out"]}
        if op == "append":
            gb.attn_append(s["cfg"], s["batch"], s["k"], s["v"], s["turns"], s["bundle"], q=s["q"], q_out=s["out"])
            return _cache_out(s, {"q": s["out"]})
        if op == "prompt":
            gb.attn_prompt(s["cfg"], s["q"], s["k"], s["v"], s["cu"], s["cu"], s["out"], s["ws"])
        else:
            gb.attn_cached(s["cfg"], s["batch"], s["q"], s["bundle"], s["out"], s["ws"])
        return {"out": s["out"]}
    if op == "rope":
        return {"q": _rotate(c, s["q"], s["pos"], s["freqs"], s["mag"]).to(s["q"].dtype),
                "k": _rotate(c, s["k"], s["pos"], s["freqs"], s["mag"]).to(s["k"].dtype)}
    if op == "append":
        seq, pos = _new_positions(s)
        page, off = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
        _store(c, s["k_pool"], s["k_scale"], _rotate(c, s["k"], pos, s["freqs"], s["mag"]), page, off)
        _store(c, s["v_pool"], s["v_scale"], s["v"].float(), page, off)
        return _cache_out(s, {"q": _rotate(c, s["q"], pos, s["freqs"], s["mag"]).to(s["q"].dtype)})
    return {"out": _plain_prompt(s) if op == "prompt" else _plain_cached(s)}


# ---------------------------------------------------------------- work, 64 bits


def work(case):
    """Inputs read once, outputs written once; products and sums of the visible
    pairs of query and key (rotations: four products and two sums a pair)."""
    c = case
    a = 4 if c["act"] == "f32" else 2
    new, lens = _shape(c)
    T, Hq, Hkv, D = sum(new), c["heads"], c["kv_heads"], c["dim"]
    cb = 1 if c.get("cache") == "e4m3" else a
    if c["op"] == "rope":
        return {"bytes": 2 * a * T * (Hq + Hkv) * D, "flops": 3 * T * (Hq + Hkv) * c["rotary"]}
    if c["op"] == "append":
        return {"bytes": T * D * (2 * a * Hq + 2 * (a + cb) * Hkv), "flops": 3 * T * (Hq + Hkv) * c["rotary"]}
    if c["op"] == "prompt":
        return {"bytes": 2 * a * T * (Hq + Hkv) * D, "flops": sum(2.0 * n * (n + 1) * D * Hq for n in new)}
    seen = [max(0, m - n + 1 + i) for n, m in zip(new, lens) for i in range(n)]
    return {"bytes": 2 * a * T * Hq * D + 2 * cb * sum(lens) * Hkv * D, "flops": 4.0 * sum(seen) * D * Hq}


def _turned64(c, x, pos):
    """Rotation as a complex product in 64 bits."""
    f, mag = _freqs(c)
    R = c["rotary"]
    ang = pos.double().view(-1, 1, 1) * torch.tensor(f, dtype=torch.float64, device=DEV)
    w = torch.polar(torch.full_like(ang, mag), ang)
    y = x.double().clone()
    i = torch.arange(R // 2, device=DEV)
    ia, ib = (i, i + R // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(y[..., ia], y[..., ib]) * w
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def _e4m3_64(x):
    """x rounded to the nearest e4m3 value, ties to the even code, in 64 bits."""
    ex = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -30))).clamp_min(-6.0)
    step = torch.exp2(ex - 3.0)
    return torch.round(x / step) * step


def _append64(c, d, which, x, new, lens):
    """Pool and scales after the append, a page at a time."""
    pool, scale = d[which + "_pool"], d[which + "_scale"]
    vals = (pool if scale is None else pool.view(torch.float8_e4m3fn)).double()
    exps = None if scale is None else scale.double() - 127.0
    table = d["table"].cpu().tolist()
    t = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        p = m - n
        while p < m:
            pg, o = table[b][p // c["page"]], p % c["page"]
            k = min(c["page"] - o, m - p)
            rows = x[t:t + k].transpose(0, 1)  # [Hkv, k, D]
            if exps is None:
                vals[pg, :, o:o + k] = rows
            else:
                e = torch.ceil(torch.log2(rows.abs().amax(dim=(1, 2)) / E4M3_MAX)).clamp(-127, 127)
                if o:
                    e = torch.maximum(e, exps[pg])
                    vals[pg, :, :o] = _e4m3_64(vals[pg, :, :o] * torch.exp2(exps[pg] - e)[:, None, None])
                vals[pg, :, o:o + k] = _e4m3_64(rows * torch.exp2(-e)[:, None, None])
                exps[pg] = e
            p, t = p + k, t + k
    return vals, None if exps is None else torch.exp2(exps)


def exact(case, seed):
    c = case
    d = _inputs(case, seed)
    new, lens = _shape(c)
    if c["op"] == "rope":
        return {w: _turned64(c, d[w], d["pos"]) for w in ("q", "k")}
    if c["op"] == "append":
        pos = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(new, lens)])
        r = {"q": _turned64(c, d["q"], pos)}
        for w, x in (("k", _turned64(c, d["k"], pos)), ("v", d["v"].double())):
            r[w + "_pool"], e = _append64(c, d, w, x, new, lens)
            if e is not None:
                r[w + "_scale"] = e
        return r
    D, G = c["dim"], c["heads"] // c["kv_heads"]
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        if c["op"] == "prompt":
            k, v = d["k"][at:at + n].double(), d["v"][at:at + n].double()
        else:
            k, v = (_wide(c, d, w, b, m) for w in ("k", "v"))
        for h in range(c["heads"]):
            kh, vh = k[:, h // G], v[:, h // G]
            for lo in range(0, n, 4096):  # rows at a time
                hi = min(n, lo + 4096)
                seen = m - n + hi  # keys that the last of these rows sees
                if seen <= 0:
                    continue
                x = d["q"][at + lo:at + hi, h].double() @ kh[:seen].T / math.sqrt(D)
                row = torch.arange(m - n + lo, m - n + hi, device=DEV)
                x.masked_fill_(torch.arange(seen, device=DEV)[None] > row[:, None], -math.inf)
                y = torch.softmax(x, -1) @ vh[:seen]
                out[at + lo:at + hi, h] = torch.where((row >= 0)[:, None], y, 0.0)
        at += n
    return {"out": out}


def _wide(c, d, which, b, m):
    """Sequence b's cached rows [m, Hkv, D] in 64 bits."""
    pages = d["table"][b, :-(-m // c["page"])].long()
    pool, scale = d[which + "_pool"], d[which + "_scale"]
    x = (pool if scale is None else pool.view(torch.float8_e4m3fn))[pages].double()
    if scale is not None:
        x = x * torch.exp2(scale[pages].double() - 127.0)[..., None, None]
    return x.transpose(1, 2).flatten(0, 1)[:m]
