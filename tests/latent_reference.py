"""Plain 64-bit forms of latent attention (torch, on the inputs' device), written from their definitions, and the
inputs that the GPU tests share."""
from __future__ import annotations

import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def prefix(v):
    return i32([0] + list(np.cumsum(v)))


def normal(seed, shape, act, sigma=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (sigma * torch.randn(shape, device="cuda", generator=g)).to(DT[act])


def apart(t):
    """The same values as part of a wider buffer of NaN: tokens (and heads) further apart, 16-byte aligned."""
    shape = [t.shape[0], *[n + 3 for n in t.shape[1:-1]], t.shape[-1] + 16]
    buf = torch.full(shape, float("nan"), dtype=t.dtype, device=t.device)
    part = (buf[:, 1:-2, 8:-8] if t.dim() == 3 else buf[:, 8:-8])
    part.copy_(t)
    return part


def heads_first(t):
    """The same [T, H, D] values with each head's tokens beside each other."""
    return t.transpose(0, 1).contiguous().transpose(0, 1)


def attention(q, k, v, n, m, scale, causal=True, present=None):
    """One sequence in 64 bits: q [n, H, K], k [m, H, K], v [m, H, V] -> out, size (sum of p |v|), lse."""
    q, k, v = q.double(), k.double(), v.double()
    j = torch.arange(m, device=q.device)[None]
    pos = torch.arange(m - n, m, device=q.device)[:, None]
    see = (j <= pos) if causal else torch.ones((n, m), dtype=torch.bool, device=q.device)
    if present is not None:
        see = see & present[None]
    none = ~see.any(1) if m else torch.ones(n, dtype=torch.bool, device=q.device)
    if m == 0:
        out = q.new_zeros((n, q.shape[1], v.shape[2]))
        return out, out.clone(), q.new_full((n, q.shape[1]), -np.inf)
    s = (torch.einsum("ihd,jhd->hij", q, k) * scale).masked_fill(~see, -np.inf)
    lse = torch.logsumexp(s, 2)
    p = torch.exp(s - lse.masked_fill(none[None], 0.0)[..., None])
    # (a value that a row does not see has no part in it, whatever it is)
    vz = torch.nan_to_num(v, 0.0, 0.0, 0.0)
    out, size = torch.einsum("hij,jhd->ihd", p, vz), torch.einsum("hij,jhd->ihd", p, vz.abs())
    return out, size, lse.T


def expanded(q, k, k_rope, v, nq, nk, scale, causal=True):
    outs, a, b = [], 0, 0
    for n, m in zip(nq, nk):
        key = k[b:b + m]
        if k_rope is not None:
            key = torch.cat((key, k_rope[b:b + m, None].expand(-1, k.shape[1], -1)), -1)
        outs.append(attention(q[a:a + n], key, v[b:b + m], n, m, scale, causal))
        a, b = a + n, b + m
    return tuple(torch.cat(x) for x in zip(*outs))


class Pool:
    """A pool of latent rows with random contents and a table of scattered pages; poison: slots that no sequence
    has written are NaN."""

    def __init__(self, seed, act, width, page, lens, poison=True, extra=2):
        rng = np.random.default_rng(seed)
        used = [-(-max(n, 0) // page) for n in lens]
        n = sum(used) + extra
        order = rng.permutation(n)
        self.page, self.lens = page, lens
        self.table = np.full((len(lens), max(1, max(used, default=0))), -1, dtype=np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = order[at:at + u]
            at += u
        self.rows = normal(seed + 1, (n, page, width), act)
        if poison:
            written = torch.zeros((n, page), dtype=torch.bool)
            for b, m in enumerate(lens):
                for i in range(used[b]):
                    written[self.table[b, i], :min(page, m - i * page)] = True
            self.rows.masked_fill_(~written.cuda()[..., None], float("nan"))

    def sequence(self, b, m):
        """Sequence b's first m rows and which of them have a page in the pool."""
        p = np.arange(m)
        ids = self.table[b, np.minimum(p // self.page, self.table.shape[1] - 1)]
        ok = (ids >= 0) & (ids < self.rows.shape[0])
        rows = self.rows[torch.from_numpy(np.where(ok, ids, 0)).long().cuda(), torch.from_numpy(p % self.page).cuda()]
        return rows, torch.from_numpy(ok).cuda()


def absorbed(q, pool, latent, nq, lens, scale, causal=True):
    outs, a = [], 0
    for b, (n, m) in enumerate(zip(nq, lens)):
        m = min(max(m, 0), pool.table.shape[1] * pool.page)
        rows, ok = pool.sequence(b, m)
        rows = rows.masked_fill(~ok[:, None], 0.0)
        key = rows[:, None].expand(-1, q.shape[1], -1)
        outs.append(attention(q[a:a + n], key, key[..., :latent], n, m, scale, causal, ok))
        a += n
    return tuple(torch.cat(x) for x in zip(*outs))


def check(out, lse, want, act, terms=2e-5):
    """Every element against its own sum. bf16: the result's rounding and the weights' (each at most 2^-8 of itself).
    fp32 scores of up to 640 products and exponentials of arguments up to about 30: errors of either sign."""
    o, size, ls = want
    bound = terms * size + 1e-30
    if act == "bf16":
        bound = bound + 1.05 * 2.0 ** -8 * (o.abs() + size)
    got = out.double()
    over = (got - o).abs() - bound
    over = torch.where(torch.isnan(over), torch.inf, over)
    assert over.max() <= 0, f"over by {float(over.max()):.2e} at {np.unravel_index(int(over.argmax()), tuple(over.shape))}"
    if lse is not None:
        empty = torch.isneginf(ls)
        assert torch.equal(torch.isneginf(lse), empty)
        assert ((lse.double() - ls).abs()[~empty] <= 1e-4).all()
