"""Plain 64-bit versions of the 8-bit attention-layer operators (numpy, CPU).

Scales and the quotients that codes come from are 32-bit numbers by definition;
both are formed here from 64-bit quotients, which round to the same 32 bits.
"""
from __future__ import annotations

import numpy as np


def quantise(x: np.ndarray):
    """(codes int8, scales float32) of the rows (last axis) of x."""
    x = np.asarray(x, dtype=np.float64)
    amax = np.max(np.abs(x), axis=-1)
    bad = ~np.isfinite(amax)
    s = (np.where(bad, 0.0, amax) / 127.0).astype(np.float32)
    live = s > 0
    div = np.where(live, s, np.float32(1)).astype(np.float64)[..., None]
    with np.errstate(over="ignore"):
        quot = (np.where(live[..., None], np.nan_to_num(x, nan=0, posinf=0, neginf=0), 0.0) / div
                ).astype(np.float32)
    q = np.clip(np.rint(quot), -127, 127).astype(np.int8)
    return q, np.where(bad, np.float32(np.nan), s)


def linear(qx, sx, qw, sw, bias=None):
    """(y, magnitude): y in 64 bits, magnitude = |scaled sum| + |bias| for error bounds."""
    S = qx.astype(np.int64) @ qw.astype(np.int64).T
    core = S * (sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :])
    b = np.zeros(len(sw)) if bias is None else bias.astype(np.float64)
    return core + b, np.abs(core) + np.abs(b)


def attention(q, k, v, lens, starts, scale, window=0):
    """Causal attention of new tokens.  q [tokens][q_heads][d]; k, v per sequence
    [len][heads][d] float64 (a NaN key or value poisons the rows that see it; keys of -inf are
    positions that the page table hides).  Returns (o, spread, logit, peak): o in 64 bits and, for
    error bounds, spread = sum_j p_j |v_j|, and per row logit = scale * max_j sum_i |q_i k_ij| and
    peak = max_j p_j max|v_j|."""
    q = np.asarray(q, dtype=np.float64)
    tokens, hq, d = q.shape
    o, spread = np.zeros(q.shape), np.zeros(q.shape)
    logit, peak = np.zeros((tokens, hq)), np.zeros((tokens, hq))
    for b, n_len in enumerate(lens):
        n = int(starts[b + 1] - starts[b])
        if n == 0 or n_len <= 0:
            continue
        kb, vb = k[b], v[b]
        g = hq // kb.shape[1]
        j = np.arange(n_len)
        for i in range(n):
            p = n_len - n + i
            seen = (j <= p) & ((j > p - window) if window else True)
            seen &= ~np.isneginf(kb[:, 0, 0])             # positions that the table hides
            if not seen.any():
                continue
            t = starts[b] + i
            for h in range(hq):
                ks, vs = kb[seen, h // g], vb[seen, h // g]
                s = (ks @ q[t, h]) * scale
                e = np.exp(s - s.max())
                w = e / e.sum()
                o[t, h] = w @ vs
                spread[t, h] = w @ np.abs(vs)
                logit[t, h] = scale * (np.abs(ks) @ np.abs(q[t, h])).max()
                peak[t, h] = (w * np.abs(vs).max(axis=1)).max()
    return o, spread, logit, peak
