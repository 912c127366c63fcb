"""Plain 64-bit versions of the 4-bit cache, attention over it, rotary positions and step plans
(numpy, CPU)."""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BAD = 255


def quantise(x: np.ndarray):
    """(codes 0 .. 15 uint8 [..., dp], scale bytes uint8 [..., groups]) of rows [..., d]; dp: d in
    whole groups of 32."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    g = -(-d // 32)
    bad = ~np.isfinite(x).all(axis=-1)
    x = np.where(bad[..., None], 0.0, np.nan_to_num(x, nan=0, posinf=0, neginf=0))
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (32 * g - d,))], axis=-1)
    x = x.reshape(x.shape[:-1] + (g, 32))
    top = np.abs(x).max(axis=-1)
    e = np.full(top.shape, -60)
    for k in range(-60, 60):                              # the least E with top <= 7 * 2^E, or 60
        e = np.where(top > 7 * 2.0 ** k, k + 1, e)
    a = np.minimum(np.abs(x) / 2.0 ** e[..., None], 6.0)
    dist = np.abs(a[..., None] - MAGNITUDES)
    best = dist.min(axis=-1, keepdims=True)
    even = np.arange(8) % 2 == 0
    # of two equally near the even one, else the nearest
    rank = np.where(dist == best, np.where(even, 0, 1), 2)
    code = rank.argmin(axis=-1) + 8 * np.signbit(x)
    code = np.where(bad[..., None, None], 0, code).astype(np.uint8)
    scale = np.where(bad[..., None], BAD, e + 127).astype(np.uint8)
    return code.reshape(code.shape[:-2] + (32 * g,)), scale


def values(code: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """Codes [..., dp] and scale bytes [..., groups] -> values [..., dp]."""
    v = MAGNITUDES[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == BAD, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def attention(q, k, v, lens, starts, scale, window=0):
    """As q8_oracle.attention, with one more number a row: mass = scale * max_j sum_i |k_ij|
    * max_i |q_i|."""
    from oracle import q8_oracle
    o, spread, logit, peak = q8_oracle.attention(q, k, v, lens, starts, scale, window)
    q = np.asarray(q, dtype=np.float64)
    mass = np.zeros(q.shape[:2])
    for b in range(len(lens)):
        if len(k[b]) == 0:
            continue
        kb = np.where(np.isfinite(k[b]), np.abs(k[b]), 0.0).sum(axis=-1).max(axis=0)  # [heads]
        rows = slice(starts[b], starts[b + 1])
        mass[rows] = scale * np.abs(q[rows]).max(axis=-1) * np.repeat(kb, q.shape[1] // len(kb))
    return o, spread, logit, peak, mass


def rotary(x, positions, frequencies, amplitude, interleaved, inverse=False):
    """x [tokens][heads][d] turned, in 64 bits."""
    x = np.array(x, dtype=np.float64)
    half = len(frequencies)
    rot = 2 * half
    p = np.asarray(positions, dtype=np.float64)
    angle = np.outer(p, frequencies) * (-1 if inverse else 1)
    c, s = (amplitude * np.cos(angle))[:, None], (amplitude * np.sin(angle))[:, None]
    i1 = np.arange(0, rot, 2) if interleaved else np.arange(half)
    i2 = i1 + 1 if interleaved else i1 + half
    a, b = x[..., i1], x[..., i2]
    y = x.copy()
    y[..., i1], y[..., i2] = a * c - b * s, b * c + a * s
    return np.where((p < 0)[:, None, None], x, y)


class Pool:
    """Sequences and pages on the host."""

    def __init__(self, sequences, width, pages, page):
        self.page, self.width = page, width
        self.held = [[] for _ in range(sequences)]
        self.lengths = [0] * sequences
        self.free = list(range(pages - 1, -1, -1))

    def plan(self, seqs, new, tokens, width=None):
        """(table, lens, starts, slots, positions, status) as cs_plan_step leaves them."""
        width = self.width if width is None else width
        n = len(seqs)
        table = np.full((n, width), -1, dtype=np.int32)
        lens, starts = np.zeros(n, np.int32), np.zeros(n + 1, np.int32)
        slots, positions = np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int32)
        empty = (table, lens, starts, slots, positions)
        most = min(width, self.width) * self.page
        total = need = 0
        for i, (s, m) in enumerate(zip(seqs, new)):
            if s == -1:
                continue
            if not 0 <= s < len(self.held) or s in list(seqs[:i]) or m < 0 or \
                    self.lengths[s] + m > most:
                return (*empty, np.array([1, i], np.int32))
            total += m
            need += -(-(self.lengths[s] + m) // self.page) - len(self.held[s])
        if total > tokens:
            return (*empty, np.array([2, total - tokens], np.int32))
        if need > len(self.free):
            return (*empty, np.array([3, need - len(self.free)], np.int32))
        t = 0
        for i, (s, m) in enumerate(zip(seqs, new)):
            if s >= 0:
                while len(self.held[s]) * self.page < self.lengths[s] + m:
                    self.held[s].append(self.free.pop())
                for p in range(self.lengths[s], self.lengths[s] + m):
                    slots[t] = self.held[s][p // self.page] * self.page + p % self.page
                    positions[t] = p
                    t += 1
                self.lengths[s] += m
                lens[i] = self.lengths[s]
                table[i, :len(self.held[s])] = self.held[s]
            starts[i + 1] = t
        return (*empty, np.zeros(2, np.int32))

    def truncate(self, seqs, lens=None):
        back = []
        for i, s in enumerate(seqs):
            to = 0 if lens is None else lens[i]
            if not 0 <= s < len(self.held) or s in list(seqs[:i]) or \
                    not 0 <= to <= self.lengths[s]:
                continue
            keep = math.ceil(to / self.page)
            back += self.held[s][keep:]
            self.held[s], self.lengths[s] = self.held[s][:keep], to
        self.free += back[::-1]
