"""Plain 64-bit forms of the attention operators on the CPU (numpy), written
from their definitions: what the GPU tests compare against."""
from __future__ import annotations

import math

import numpy as np


def frequencies(R, base=10000.0):
    return np.array([base ** (-2.0 * i / R) for i in range(R // 2)])


def rotate(x, positions, freqs, layout, mag=1.0, sign=1.0):
    """x [T, H, D]: its first 2 * len(freqs) elements turned."""
    y = np.array(x, dtype=np.float64)
    n = len(freqs)
    ang = sign * np.asarray(positions, dtype=np.float64)[:, None] * freqs
    c, s = (mag * np.cos(ang))[:, None], (mag * np.sin(ang))[:, None]
    ia = np.arange(n) if layout == "half" else 2 * np.arange(n)
    ib = ia + (n if layout == "half" else 1)
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def e4m3_round(x):
    """Nearest e4m3 value, ties to even, +-448 beyond."""
    a = np.minimum(np.abs(np.asarray(x, dtype=np.float64)), 448.0)  # (a NaN stays)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -40))), -6.0)
    step = 2.0 ** (e - 3)
    return np.copysign(np.round(a / step) * step, x)


def e4m3_values():
    """Value of each of the 256 codes."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = math.nan if (c & 127) == 127 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        v[c] = -mag if c & 128 else mag
    return v


def append(vals, exps, x, new, lens, table, page):
    """x [T, Hkv, D] into vals [pages, Hkv, page, D] (code values and exponents, or plain values with exps None), in place."""
    t = 0
    n_pages = vals.shape[0]
    for b, (n, m) in enumerate(zip(new, lens)):
        done = 0
        while done < n:
            p = m - n + done
            pg, off = p // page, p % page
            k = min(page - off, n - done)
            rows = np.swapaxes(x[t + done:t + done + k], 0, 1)
            done += k
            if pg < 0 or pg >= table.shape[1] or not 0 <= table[b, pg] < n_pages:
                continue
            i = table[b, pg]
            if exps is None:
                vals[i, :, off:off + k] = rows
                continue
            for h in range(vals.shape[1]):
                fin = np.abs(rows[h][np.isfinite(rows[h])])
                top = float(fin.max()) if fin.size else 0.0
                e = -127
                if top > 0:
                    f, ex = math.frexp(top)
                    e = max(ex - 9 + (f > 0.875), -127)
                if off > 0:
                    old = int(exps[i, h])
                    e = max(e, old)
                    vals[i, h, :off] = e4m3_round(vals[i, h, :off] * 2.0 ** (old - e))
                vals[i, h, off:off + k] = e4m3_round(rows[h] * 2.0 ** -e)
                exps[i, h] = e
        t += n


def attention(q, keys, values, pos, scale, causal=True, window=0, present=None):
    """One sequence: q [n, Hq, D] at positions pos [n], keys and values [m, Hkv, D]; (out, lse)."""
    n, Hq, D = q.shape
    m, Hkv = keys.shape[0], keys.shape[1]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    j = np.arange(m)
    for i in range(n):
        see = np.ones(m, dtype=bool) if present is None else present.copy()
        if causal:
            see &= j <= pos[i]
        if window > 0:
            see &= j > pos[i] - window
        if not see.any():
            continue
        for h in range(Hq):
            s = (keys[see, h // (Hq // Hkv)] @ q[i, h]) * scale
            top = s.max()
            p = np.exp(s - top)
            out[i, h] = p @ values[see, h // (Hq // Hkv)] / p.sum()
            lse[i, h] = top + math.log(p.sum())
    return out, lse
