"""Calls of more workgroups than one grid dimension takes (2^32 threads), up to the row counts that
the interface states: nothing is refused, and the last rows are right."""
from __future__ import annotations

import pytest
import torch

from oracle import q8_oracle as o8
from paper_2112_13896_amd import ops
from tests.q8_util import f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()                                 # tens of GB


@pytest.mark.parametrize("rows,c", [((1 << 26) + 5, 3), ((1 << 24) + 3, 1025)])
def test_quantise_rows(rows, c):
    """A wavefront a row, and four."""
    x = torch.empty((rows, c), dtype=torch.float16, device="cuda").normal_()
    q = torch.full((rows, c), -128, dtype=torch.int8, device="cuda")   # no code
    ops.quantise_rows(x, q=q, scale=(s := torch.full((rows,), -1.0, device="cuda")))
    assert not bool((s < 0).any()) and not any(bool((p == -128).any()) for p in q.split(1 << 22))
    for first in (0, rows // 2, (rows >> 22 << 22) - 50, rows - 100):
        rq, rs = o8.quantise(f64(x[first:first + 100]))
        assert (q[first:first + 100].cpu().numpy() == rq).all()
        assert (s[first:first + 100].cpu().numpy() == rs).all()


def _linear(rows, k, d_out, out_dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.empty((rows, k), dtype=torch.int8, device="cuda")
    for part in x.split(1 << 26):
        part.random_(-127, 128, generator=g)
    w = torch.randint(-127, 128, (d_out, k), dtype=torch.int8, device="cuda", generator=g)
    sx, sw = torch.full((rows,), 0.5, device="cuda"), torch.full((d_out,), 0.25, device="cuda")
    out = torch.full((rows, d_out), float("nan"), dtype=out_dtype, device="cuda")
    ops.linear_q8(x, w, sw, sx=sx, out_dtype=out_dtype, out=out,
                  ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert not any(bool(torch.isnan(p).any()) for p in out.split(1 << 27))
    for first in (0, rows // 2, (rows >> 22 << 22) - 50, rows - 100):
        want = (x[first:first + 100].cpu().long() @ w.cpu().long().t()).double() * 0.125
        assert torch.equal(out[first:first + 100].cpu(), want.to(out_dtype))


def test_linear_of_rows_that_start_anywhere():
    _linear((1 << 30) + 77, 1, 1, torch.float16)


def test_linear_tiles():
    _linear((1 << 31) - 1, 16, 1, torch.float16)


def test_cache():
    """One token of many is kept, and read back among slots that are not in the cache."""
    heads, d, page = 16, 16, 16
    tokens = (1 << 24) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((1, heads, d), generator=g, device="cuda").half() for _ in range(2))
    cache = ops.PagedCache.empty(1, heads, page, d)
    slots = torch.full((tokens,), -1, device="cuda")
    slots[-1] = 7
    ops.cache_write(cache, k.expand(tokens, heads, d), v.expand(tokens, heads, d), slots)
    for x, y in zip((k, v), ops.cache_read(cache, slots, torch.float16)):
        q, s = o8.quantise(f64(x))
        want = torch.from_numpy(q.astype("float32") * s[..., None]).half()
        assert torch.equal(y[-1:].cpu(), want)
        assert not any(bool(p.any()) for p in y[:-1].split(1 << 20))


def test_attention():
    """Many sequences of one token each, many heads: a token's output is its value."""
    batch, heads, d, page, pages = 4096, 4096, 16, 16, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = ops.PagedCache.empty(pages, heads, page, d)
    for t in (cache.k, cache.v):
        t.random_(-127, 128, generator=g)
    cache.k_scale.fill_(0.5)
    cache.v_scale.fill_(0.25)
    q = torch.randn((batch, heads, d), generator=g, device="cuda")
    table = torch.randint(0, pages, (batch, 1), dtype=torch.int32, device="cuda", generator=g)
    plan = ops.paged_attention_plan(q.dtype, heads, page, d, batch, heads, batch, 1, 1)
    assert plan["workgroups"] > 1 << 24
    out = ops.paged_attention(q, cache, table, torch.ones(batch, dtype=torch.int32, device="cuda"),
                              torch.arange(batch + 1, dtype=torch.int32, device="cuda"), max_len=1)
    want = cache.v[:, :, 0].float() * 0.25
    assert torch.allclose(out, want[table[:, 0].long()], rtol=2.0 ** -20, atol=0)


@pytest.mark.parametrize("c", [(1 << 31) - 1, (1 << 31) - 8])
def test_quantise_the_longest_row(c):
    x = torch.zeros((1, c), dtype=torch.float16, device="cuda")
    x[0, ::1000003] = 3.0
    x[0, -9:] = torch.tensor([1.0, -4, 2, 254, -127, 0, 0.5, 64, -254], device="cuda").half()
    x[0, :3] = torch.tensor([100.0, -1, 253], device="cuda").half()
    q = torch.full((1, c), -128, dtype=torch.int8, device="cuda")
    _, s = ops.quantise_rows(x, q=q)
    assert s.tolist() == [2.0]
    assert q[0, :3].tolist() == [50, 0, 126] and q[0, -9:].tolist() == [0, -2, 1, 127, -64, 0, 0, 32, -127]
    assert not any(bool((p == -128).any()) for p in q[0].split(1 << 28))
    assert int(q[0, 3:-9].count_nonzero()) == len(range(1000003, c - 9, 1000003))
