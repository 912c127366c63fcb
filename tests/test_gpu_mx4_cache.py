"""The paged 4-bit cache: codes and scales as defined, to the byte, and read back as they stand."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as o4
from paper_2112_13896_amd import ops
from tests.mx4_util import (DTYPES, f64, pack_keys, pack_value_scales, pack_values, rand)

pytestmark = pytest.mark.gpu


def _expect(k, v, slots, pages, page, fill):
    """The cache's four arrays after a write into arrays of `fill` bytes."""
    tokens, heads, d = k.shape
    g = -(-d // 32)
    code = {n: np.full((pages, heads, page, 32 * g), fill & 15, np.uint8) for n in "kv"}
    scale = {n: np.full((pages, heads, page, g), fill, np.uint8) for n in "kv"}
    for n, x in (("k", k), ("v", v)):
        c, s = o4.quantise(f64(x))
        for t in range(tokens):
            if 0 <= slots[t] < pages * page:
                pg, off = divmod(int(slots[t]), page)
                code[n][pg, :, off], scale[n][pg, :, off] = c[t], s[t]
    return (pack_keys(code["k"]), pack_values(code["v"]), scale["k"],
            pack_value_scales(scale["v"]))


def _written(k, v, slots, pages, page, fill=0x55):
    heads, d = k.shape[1:]
    cache = ops.PagedCache4.empty(pages, heads, page, d)
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.fill_(fill)
    ops.cache_write(cache, k, v, torch.as_tensor(slots).cuda())
    return cache


def _check(k, v, slots, pages, page):
    cache = _written(k.cuda(), v.cuda(), slots, pages, page)
    for got, want, name in zip((cache.k, cache.v, cache.k_scale, cache.v_scale),
                               _expect(k, v, slots, pages, page, 0x55),
                               ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(got.cpu().numpy(), want), name
    return cache


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,heads,d,page", [(1, 1, 16, 16), (3, 5, 48, 16), (37, 2, 80, 32),
                                                 (130, 8, 128, 64), (21, 3, 256, 1024),
                                                 (18, 1, 144, 16)])
def test_written_bytes(dtype, tokens, heads, d, page):
    r = np.random.default_rng(tokens)
    pages = -(-tokens // page) + 2
    k, v = (rand(r, (tokens, heads, d), DTYPES[dtype], 3.0) for _ in "kv")
    slots = r.permutation(pages * page)[:tokens].astype(np.int64)
    _check(k, v, slots, pages, page)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_and_borders_of_scales(dtype):
    """Values on the borders between codes, at the largest that a scale takes and just past it, at
    both ends of the scales, zeros of both signs."""
    dt = DTYPES[dtype]
    rows = []
    for e in (0, -1, 5, -12):
        rows.append(2.0 ** e * np.array([7, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25,
                                         -1.75, -2.5, -3.5, -5, -7]))
    for top in (7.0, 7.03125, 6.96875, 3.5, 3.515625, 1e-30, 1e-45, 2.0 ** -62, 2.0 ** -61, 1e30,
                3e38, 6 * 2.0 ** 60, 65504.0, 2.0 ** -24, 0.0):
        rows.append(top * np.linspace(-1, 1, 16))
    x = torch.from_numpy(np.tile(np.stack(rows), (1, 3))).to(dt)
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).view(len(rows), 1, 48)
    _check(x, -x, np.arange(len(rows)), 2, 16)


def test_scales_of_every_exponent():
    """fp32 rows of magnitudes from the smallest to the largest numbers there are."""
    e = np.arange(-149, 128)
    r = np.random.default_rng(0)
    x = np.ldexp(r.uniform(1, 2, (len(e), 1, 32)) * r.choice([-1, 1], (len(e), 1, 32)), e[:, None,
                                                                                       None])
    x = torch.from_numpy(x.astype(np.float32))
    assert torch.isfinite(x).all()
    _check(x, x, np.arange(len(e)), 18, 16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [32, 80, 128, 256])
def test_rows_that_are_not_finite(dtype, d):
    """All of a row, and no other row, is NaN."""
    r = np.random.default_rng(d)
    k, v = (rand(r, (9, 3, d), DTYPES[dtype]) for _ in "kv")
    k[2, 1, d - 1], k[3, 0, 0], v[4, 2, 5], v[5, 0, d // 2] = np.nan, np.inf, -np.inf, np.nan
    cache = _check(k, v, np.arange(9), 1, 16)
    gk, gv = ops.cache_read(cache, torch.arange(9).cuda(), torch.float32)
    for got, x in ((gk, k), (gv, v)):
        bad = ~torch.isfinite(x).all(dim=-1)
        assert torch.isnan(got.cpu()[bad]).all() and torch.isfinite(got.cpu()[~bad]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_alignment(dtype):
    """Tokens and heads apart, heads before tokens, rows that start anywhere: the same bytes."""
    dt = DTYPES[dtype]
    r = np.random.default_rng(5)
    qkv = rand(r, (11, 7, 64), dt).cuda()
    slots = torch.arange(11).cuda()
    k, v = qkv[:, 2:4], qkv[:, 5:7]
    want = _written(k.contiguous(), v.contiguous(), slots, 1, 16)
    odd = torch.zeros(11 * 150 + 7, dtype=dt, device="cuda")
    apart = odd[3:3 + 11 * 150].view(11, 150)[:, :2 * 67].view(11, 2, 67)[:, :, 1:65]
    apart.copy_(k)
    turned = v.transpose(0, 1).contiguous().transpose(0, 1)
    for a, b in ((k, v), (apart, v), (k, turned), (apart, turned)):
        got = _written(a, b, slots, 1, 16)
        for n in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(got, n), getattr(want, n)), n


def test_slots_outside_the_cache():
    r = np.random.default_rng(6)
    k, v = (rand(r, (6, 2, 32), torch.bfloat16) for _ in "kv")
    slots = np.array([3, -1, 32, 2 ** 40, -2 ** 62, 31], dtype=np.int64)
    cache = _check(k, v, slots, 2, 16)
    got = ops.cache_read(cache, torch.from_numpy(slots).cuda(), torch.float16)
    for t in got:
        assert not t[1:5].any() and t[0].any() and t[5].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", range(16, 257, 48))
def test_read_back(dtype, d):
    """Any order, repeats; each value is its code times its scale, rounded once to the type."""
    dt = DTYPES[dtype]
    r = np.random.default_rng(d)
    x = torch.from_numpy(r.standard_normal((2, 50, 3, d)) *
                         np.exp(r.standard_normal((2, 50, 3, 1))))
    x = x.to(dt)
    cache = _written(x[0].cuda(), x[1].cuda(), np.arange(50) + 7, 4, 16)
    slots = r.integers(0, 50, size=77)
    got = ops.cache_read(cache, torch.from_numpy(slots + 7).cuda(), dt)
    for g, src in zip(got, x):
        want = o4.values(*o4.quantise(f64(src)))[slots][..., :d]
        assert torch.equal(g.cpu(), torch.from_numpy(want).to(dt))


def test_no_tokens():
    cache = ops.PagedCache4.empty(1, 2, 16, 32)
    none = torch.empty((0, 2, 32), device="cuda")
    slots = torch.empty((0,), dtype=torch.int64, device="cuda")
    ops.cache_write(cache, none, none, slots)
    k, v = ops.cache_read(cache, slots, torch.float32)
    assert k.shape == v.shape == (0, 2, 32)
