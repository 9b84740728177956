"""fp64 NumPy reference of the operators over a long memory: norm and rotation
of queries and keys, the paged cache with its quantised formats, and attention
of a chunk of new tokens over it.  Written for clarity, one row at a time;
shares no code with the library."""
from __future__ import annotations

import numpy as np

TOP = {"int8": 127.0, "fp8": 448.0}


def rope_table(n_positions, rotary, theta=10000.0):
    """float64 [n_positions][rotary / 2][2] = (cos, sin)."""
    inv = theta ** (-np.arange(0, rotary, 2) / rotary)
    a = np.arange(n_positions)[:, None] * inv[None]
    return np.stack([np.cos(a), np.sin(a)], -1)


def norm_rope(x, gain, table, positions, pairs, eps):
    """x [rows][heads][dh]; gain [dh] or None; table [positions][r/2][2] or
    None; eps None: no norm."""
    y = np.array(x, np.float64)
    if eps is not None:
        y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + eps) * (1.0 if gain is None else np.asarray(gain, np.float64))
    if table is None:
        return y
    out = y.copy()
    half = table.shape[1]
    for i in range(half):
        a, b = (i, i + half) if pairs == "halves" else (2 * i, 2 * i + 1)
        c, s = (table[positions, i, j].astype(np.float64)[:, None] for j in (0, 1))
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def e4m3(y):
    """Nearest value with 3 bits behind the leading one, smallest normal 2^-6,
    ties to even (|y| <= 448)."""
    y = np.asarray(y, np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.rint(y / step) * step


def quantise(x, fmt):
    """(codes as values, scale [...]) of rows x [...][dh]."""
    x = np.asarray(x, np.float64)
    s = np.max(np.abs(x), -1) / TOP[fmt]
    bad = ~np.isfinite(x).all(-1)
    y = np.where((s > 0)[..., None] & ~bad[..., None], x, 0.0) / np.where((s > 0) & ~bad, s, 1.0)[..., None]
    return (np.rint(y) if fmt == "int8" else e4m3(y)), np.where(bad, np.nan, s)


def place(page_table, page_size, seq, pos):
    """(page, slot) of a position of a sequence."""
    return int(page_table[seq][pos // page_size]), pos % page_size


def gather(k, v, k_scale, v_scale, page_table, seq, length):
    """Keys and values [length][heads][dh] of a sequence from the cache's
    arrays k [pages][heads][slots][dh], v [pages][heads][dh][slots]."""
    heads, size, dh = k.shape[1:]
    ks, vs = np.zeros((length, heads, dh)), np.zeros((length, heads, dh))
    for pos in range(length):
        pg, sl = place(page_table, size, seq, pos)
        ks[pos], vs[pos] = k[pg, :, sl], v[pg, :, :, sl]
        if k_scale is not None:
            ks[pos] *= k_scale[pg, :, sl][:, None]
            vs[pos] *= v_scale[pg, :, sl][:, None]
    return ks, vs


def attend(q, k, v, start, scale, causal=False, window=0, cap=0.0, slopes=None, prefix=0):
    """One sequence: q [rows][heads][dh] at positions start .., k and v
    [keys][kv_heads][dh].  Returns (out, lse)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, heads, dh = q.shape
    keys, group = k.shape[0], heads // max(1, k.shape[1])
    out, lse = np.zeros((n, heads, dh)), np.full((n, heads), -np.inf)
    for i in range(n):
        p = start + i
        j = np.arange(keys)
        near = np.ones(keys, bool)
        if causal:
            near &= j <= p
        if window:
            near &= np.abs(p - j) < window
        see = np.nonzero(near | (j < prefix))[0]
        if see.size == 0:
            continue
        for h in range(heads):
            with np.errstate(invalid="ignore", over="ignore"):
                z = scale * (k[see, h // group] @ q[i, h])
                if cap > 0:
                    z = cap * np.tanh(z / cap)
                if slopes is not None:
                    z = z - slopes[h] * np.abs(p - see)
                top = np.max(z)
                w = np.exp(z - top)
                lse[i, h] = top + np.log(np.sum(w))
                out[i, h] = (w / np.sum(w)) @ v[see, h // group]
    return out, lse
