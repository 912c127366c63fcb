"""Cases and error bounds shared by the tests of the 4-bit cache and attention over it."""
from __future__ import annotations

import numpy as np
import torch

from oracle import mx4_oracle as o4
from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, ROUND, f64, rand  # noqa: F401

# A query's pieces: how far an element is held, of the row's largest.  bf16: two e4m3 pieces of a
# row whose largest is at least 2^7, the second in units of 2^-4 and e4m3's steps at least 2^-9, so
# half a step is 2^-14.  Otherwise e2m3 pieces of a row whose largest is in [3.5, 7): the first is
# off by 2^-2, the second by 2^-3 in units of 2^-4, the others by 2^-4 in units of 2^-8, 2^-13,
# 2^-18.  Four: 2^-17 / 3.5; five: 2^-22 / 3.5.
QUERY = {torch.bfloat16: 2.0 ** -21, torch.float16: 2.0 ** -18.8, torch.float32: 2.0 ** -23.8}
PIECES = {torch.bfloat16: 2, torch.float16: 4, torch.float32: 5}


def pack_keys(code):
    """Codes [pages][heads][page][dp] -> bytes [pages][heads][page][dp / 2]."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def pack_values(code):
    """Codes [pages][heads][page][dp] -> bytes [pages][heads][page / 4][dp / 8][4][4]."""
    p, h, n, dp = code.shape
    b = pack_keys(code).reshape(p, h, n // 4, 4, dp // 8, 4)
    return np.ascontiguousarray(b.transpose(0, 1, 2, 4, 3, 5))


def pack_value_scales(s):
    """[pages][heads][page][groups] -> [pages][heads][page / 4][groups][4]."""
    p, h, n, g = s.shape
    return np.ascontiguousarray(s.reshape(p, h, n // 4, 4, g).transpose(0, 1, 2, 4, 3))


def bound_attention(o, spread, logit, peak, mass, length, d, dtype, one_piece=False):
    """Output rounding, plus the weights' error times sum_j p_j |v_j|.  Values are exact in bf16.
    A weight is the sum of bf16 pieces, each rounding what the others leave to half a step, 2^-8 of
    it: two for 16-bit outputs (2^-16), three for fp32 (2^-24), one where the plan takes 128 rows
    of bf16 (2^-8).  A logit: the query's pieces (QUERY), and a sum of d products for each piece,
    rounded to at most 2^-23 of the sum of magnitudes at each; exp doubles it for the numerator's
    and the denominator's share, and its own argument, below 2^8 in log2 units where it counts, is
    rounded to 2^-24 of that, its result to 2^-22.  Sums of weights: at most length / 16 + 64 adds
    deep.  Pieces of bf16 have the exponents of 32-bit floats, so nothing is lost at the low end but
    weights below 2^-126 of the largest: 2^-100 of the row's largest part covers `length` of them."""
    rel, tiny = ROUND[dtype]
    weight = 2.0 ** -8 if one_piece else 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -16
    dl = (d * PIECES[dtype] + 8) * 2.0 ** -23 * logit + QUERY[dtype] * mass
    dl = dl[..., None] + 2.0 ** -16
    depth = (length / 16 + 64) * 2.0 ** -24 + 2.0 ** -21
    return rel * np.abs(o) + (weight + 2 * dl + depth) * spread + 2.0 ** -100 * peak[..., None] + \
        tiny


class Sequences:
    """Sequences of new tokens over a paged 4-bit cache: everything on the CPU, made from a seed.
    `seqs`: list of (new tokens, tokens in the cache with them)."""

    def __init__(self, seed, seqs, heads, group, d, page, dtype, amp=1.0, pad_tokens=0,
                 spare_pages=3):
        r = np.random.default_rng(seed)
        self.seqs, self.heads, self.group, self.d, self.page = seqs, heads, group, d, page
        self.dtype = dtype
        n_new = sum(n for n, _ in seqs)
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.lens = np.array([m for _, m in seqs], dtype=np.int32)
        self.q = rand(r, (n_new + pad_tokens, heads * group, d), dtype, amp)
        per = [-(-max(m, 0) // page) for _, m in seqs]
        self.pages = sum(per) + spare_pages
        order = r.permutation(self.pages)
        self.table = np.full((len(seqs), max(1, max(per))), -7, dtype=np.int32)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.pages, heads, page, d)
        self.kc, self.ks = o4.quantise(r.standard_normal(shape))
        self.vc, self.vs = o4.quantise(r.standard_normal(shape) *
                                       np.exp(0.5 * r.standard_normal(shape[:3]))[..., None])
        # what no sequence holds must not matter: NaN rows everywhere outside the sequences
        live = np.zeros((self.pages, page), dtype=bool)
        for b, (_, m) in enumerate(seqs):
            for j in range(max(m, 0)):
                live[self.table[b, j // page], j % page] = True
        pg, off = np.nonzero(~live)
        for h in range(heads):
            self.spoil("k", pg, h, off)
            self.spoil("v", pg, h, off)

    def spoil(self, which, page, head, off):
        """Rows that were not finite when written."""
        getattr(self, which + "c")[page, head, off] = 0
        getattr(self, which + "s")[page, head, off] = o4.BAD

    def slot(self, b, j):
        return int(self.table[b, j // self.page]) * self.page + j % self.page

    def dense(self):
        """Per sequence keys and values [len][heads][d] in 64 bits (keys -inf where the table
        names no page of the cache)."""
        ks, vs = [], []
        for b, (_, m) in enumerate(self.seqs):
            j = np.arange(max(m, 0))
            pg, off = self.table[b][j // self.page], j % self.page
            ok = (pg >= 0) & (pg < self.pages)
            pg = np.where(ok, pg, 0)
            k = o4.values(self.kc[pg, :, off], self.ks[pg, :, off])[..., :self.d]
            v = o4.values(self.vc[pg, :, off], self.vs[pg, :, off])[..., :self.d]
            k[~ok], v[~ok] = -np.inf, 0.0
            ks.append(k)
            vs.append(v)
        return ks, vs

    def cache(self, device="cuda"):
        return ops.PagedCache4(*(torch.from_numpy(np.ascontiguousarray(a)).to(device) for a in (
            pack_keys(self.kc), pack_values(self.vc), self.ks, pack_value_scales(self.vs))),
            d=self.d)

    def args(self, device="cuda"):
        return (self.q.to(device), self.cache(device), torch.from_numpy(self.table).to(device),
                torch.from_numpy(self.lens).to(device), torch.from_numpy(self.starts).to(device))

    def check(self, out, scale=None, window=0, what="", max_len=None):
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        k, v = self.dense()
        *ref, mass = o4.attention(f64(self.q), k, v, self.lens, self.starts,
                                  float(np.float32(scale)), window)
        got = f64(out)
        nan = np.isnan(ref[0])
        assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places than expected"
        longest = int(max(1, self.lens.max()))
        rows = ops.paged_attention_plan(self.dtype, self.heads, self.page, self.d, len(self.q),
                                        self.heads * self.group, len(self.seqs),
                                        self.table.shape[1], max_len, window, bits=4)["rows"]
        one = rows == 128 and self.dtype == torch.bfloat16
        tol = bound_attention(*ref, mass, longest, self.d, self.dtype, one)
        err = np.abs(got - ref[0])
        bad = ~nan & ~(err <= tol)
        if bad.any():
            i = tuple(np.argwhere(bad)[0])
            raise AssertionError(f"{what}: {bad.sum()} outputs out of tolerance, first at {i}: "
                                 f"{got[i]!r} for {ref[0][i]!r}, bound {tol[i]!r}")
        return float(np.max(np.where(nan, 0, err / tol), initial=0.0))
