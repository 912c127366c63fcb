"""Row quantisation and the paged 8-bit cache against the 64-bit oracle: codes, scales and
values read back are equal bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import q8_oracle as o8
from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, f64, rand

pytestmark = pytest.mark.gpu


def _check_rows(x, q, s):
    rq, rs = o8.quantise(f64(x))
    assert np.array_equal(s.cpu().numpy().view(np.uint32), rs.view(np.uint32)) or \
        np.array_equal(s.cpu().numpy(), rs, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), rq)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,c", [(1, 1), (1, 16), (3, 7), (5, 64), (17, 100), (1, 2048),
                                    (4, 2049), (9, 2055), (2, 8192), (3, 10007), (1000, 512)])
def test_rows(dtype, rows, c):
    r = np.random.default_rng(rows * 31 + c)
    x = rand(r, (rows, c), DTYPES[dtype])
    q, s = ops.quantise_rows(x.cuda())
    _check_rows(x, q, s)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_and_extremes(dtype):
    """Quotients at and next to half way between two codes, zero rows, the type's largest and
    smallest numbers."""
    dt = DTYPES[dtype]
    fi = torch.finfo(dt)
    half = torch.arange(-127, 128, dtype=torch.float32) + 0.5
    rows = [torch.cat([torch.tensor([127.0]), half[1:-1]]),            # scale 1
            torch.cat([torch.tensor([1.0]), half[1:-1] / 128]),
            torch.cat([torch.tensor([254.0]), half[1:-1] * 2]),
            torch.zeros(254), -torch.zeros(254),
            torch.full((254,), fi.max), torch.full((254,), -fi.max),
            torch.full((254,), fi.tiny), torch.full((254,), fi.smallest_normal) * half[:254] / 128]
    x = torch.stack([t[:254] for t in rows]).to(dt)
    if dt == torch.float32:
        sub = torch.zeros(254)
        sub[:5] = torch.tensor([190.0, 1.0, -64.0, 100.0, 189.0]) * 2.0 ** -149
        x = torch.cat([x, sub[None], (half[:254] * 2.0 ** -130)[None]])
        near = torch.nextafter(half[:254] * 3, torch.tensor(0.0))
        near[0] = 381.0
        x = torch.cat([x, near[None]])
    q, s = ops.quantise_rows(x.cuda())
    _check_rows(x, q, s)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(bad):
    x = rand(np.random.default_rng(1), (6, 300), torch.float32)
    x[2, 299] = bad
    x[4, 0] = bad
    q, s = ops.quantise_rows(x.cuda())
    _check_rows(x, q, s)
    assert torch.isnan(s).cpu().tolist() == [False, False, True, False, True, False]


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_offsets(dtype):
    """Row strides and starts that no vector load can take, and a destination of any stride whose
    padding is left alone."""
    dt = DTYPES[dtype]
    r = np.random.default_rng(8)
    big = rand(r, (7, 203), dt).cuda()
    for x in (big[:, 1:131], big[1:, 3:], big[::2, :64], big[:, :200]):
        q, s = ops.quantise_rows(x)
        _check_rows(x, q, s)
        buf = torch.full((x.shape[0], x.shape[1] + 5), 99, dtype=torch.int8, device="cuda")
        q2, s2 = ops.quantise_rows(x, q=buf[:, 2:2 + x.shape[1]])
        assert torch.equal(q2, q) and torch.equal(s2, s)
        assert bool((buf[:, :2] == 99).all()) and bool((buf[:, 2 + x.shape[1]:] == 99).all())


def test_no_rows():
    q, s = ops.quantise_rows(torch.empty((0, 8), device="cuda"))
    assert q.shape == (0, 8) and s.shape == (0,)


# ------------------------------------------------------------------ cache
def _as_type(v64, dt):
    """code * scale in 32 bits, rounded once to the type."""
    return torch.from_numpy(v64.astype(np.float32)).to(dt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,d,page,tokens", [(1, 16, 16, 1), (3, 80, 16, 37), (8, 128, 64, 200),
                                                 (2, 256, 1024, 5), (5, 144, 32, 64)])
def test_write_then_read(dtype, heads, d, page, tokens):
    dt = DTYPES[dtype]
    r = np.random.default_rng(heads * 1000 + d)
    pages = -(-tokens // page) + 2
    cache = ops.PagedCache.empty(pages, heads, page, d)
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.fill_(77)
    k, v = rand(r, (tokens, heads, d), dt, 3.0), rand(r, (tokens, heads, d), dt)
    slots = torch.from_numpy(r.permutation(pages * page)[:tokens].astype(np.int64))
    drop = {0: -1, tokens // 2: pages * page, tokens - 1: 2 ** 40} if tokens > 4 else {}
    for i, s in drop.items():
        slots[i] = s
    ops.cache_write(cache, k.cuda(), v.cuda(), slots.cuda())
    want = {n: np.full(t.shape, 77, dtype=np.int8 if i < 2 else np.float32)
            for i, (n, t) in enumerate((("k", cache.k), ("v", cache.v), ("ks", cache.k_scale),
                                        ("vs", cache.v_scale)))}
    for x, c, s in ((k, "k", "ks"), (v, "v", "vs")):
        rq, rs = o8.quantise(f64(x))
        for i in range(tokens):
            if i not in drop:
                p, off = divmod(int(slots[i]), page)
                want[c][p, :, off], want[s][p, :, off] = rq[i], rs[i]
    assert np.array_equal(cache.k.cpu().numpy(), want["k"])
    assert np.array_equal(cache.v.cpu().numpy(), want["v"])
    assert np.array_equal(cache.k_scale.cpu().numpy(), want["ks"])
    assert np.array_equal(cache.v_scale.cpu().numpy(), want["vs"])
    again = torch.cat([slots, slots.flip(0)])               # any order, repeats
    got = ops.cache_read(cache, again.cuda(), dt)
    for out, c, s in zip(got, ("k", "v"), ("ks", "vs")):
        ref = np.zeros((2 * tokens, heads, d))
        for i, sl in enumerate(again.tolist()):
            if 0 <= sl < pages * page:
                p, off = divmod(sl, page)
                ref[i] = want[c][p, :, off].astype(np.float64) * want[s][p, :, off][:, None]
        assert torch.equal(out.cpu(), _as_type(ref, dt))


@pytest.mark.parametrize("dtype", DTYPES)
def test_write_strided(dtype):
    """Keys and values as slices of one projection's output, at an odd element too."""
    dt = DTYPES[dtype]
    heads, d, tokens, page = 3, 48, 21, 16
    r = np.random.default_rng(4)
    for lead in (0, 8, 5):
        x = rand(r, (tokens, lead + 2 * heads * d + 8), dt).cuda()
        k = x[:, lead:lead + heads * d].unflatten(1, (heads, d))
        v = x[:, lead + heads * d:lead + 2 * heads * d].unflatten(1, (heads, d))
        slots = torch.arange(tokens, device="cuda")
        a, b = ops.PagedCache.empty(2, heads, page, d), ops.PagedCache.empty(2, heads, page, d)
        ops.cache_write(a, k, v, slots)
        ops.cache_write(b, k.contiguous(), v.contiguous(), slots)
        for t, u in zip(ops.cache_read(a, slots, dt), ops.cache_read(b, slots, dt)):
            assert torch.equal(t, u)
        by_head = k.transpose(0, 1).contiguous().transpose(0, 1)    # head-major storage
        ops.cache_write(a, by_head, v, slots)
        assert torch.equal(ops.cache_read(a, slots, dt)[0], ops.cache_read(b, slots, dt)[0])


def test_write_not_finite():
    """A token's head with a NaN reads back as NaN; its other heads and tokens are as ever."""
    r = np.random.default_rng(5)
    k, v = rand(r, (4, 2, 32), torch.float32), rand(r, (4, 2, 32), torch.float32)
    k[1, 0, 7], v[2, 1, 31] = float("nan"), float("inf")
    cache = ops.PagedCache.empty(1, 2, 16, 32)
    slots = torch.arange(4, device="cuda")
    ops.cache_write(cache, k.cuda(), v.cuda(), slots)
    rk, rv = ops.cache_read(cache, slots, torch.float32)
    nan_k, nan_v = torch.isnan(rk).all(-1).cpu(), torch.isnan(rv).all(-1).cpu()
    assert nan_k.nonzero().tolist() == [[1, 0]] and nan_v.nonzero().tolist() == [[2, 1]]
    assert torch.isnan(rk).any(-1).cpu().nonzero().tolist() == [[1, 0]]


def test_offsets_past_32_bits():
    """The last page of a cache whose arrays are larger than 4 GiB."""
    heads, d, page = 16, 256, 1024
    pages = (1 << 32) // (heads * d * page) + 3
    cache = ops.PagedCache.empty(pages, heads, page, d)
    r = np.random.default_rng(6)
    k, v = rand(r, (20, heads, d), torch.bfloat16), rand(r, (20, heads, d), torch.bfloat16)
    slots = torch.arange(pages * page - 20, pages * page)
    ops.cache_write(cache, k.cuda(), v.cuda(), slots.cuda())
    got = ops.cache_read(cache, slots.cuda(), torch.float32)
    for x, y in zip((k, v), got):
        q, s = o8.quantise(f64(x))
        assert np.array_equal(y.cpu().numpy(), q.astype(np.float32) * s[..., None])
