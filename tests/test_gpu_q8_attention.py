"""Paged attention over the 8-bit cache against the 64-bit oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, Sequences, f64

pytestmark = pytest.mark.gpu

# (new tokens, positions with them): lengths of one and zero, ends inside tiles and pages,
# fewer positions than new tokens (rows that see nothing), sequences without new tokens
ONE = [(1, 1), (1, 2), (1, 16), (1, 17), (1, 33), (1, 64), (1, 65), (1, 200), (1, 0), (0, 50),
       (1, 127)]
DRAFT = [(5, 5), (3, 40), (8, 129), (2, 1), (1, 300), (4, 0), (0, 0)]
CHUNK = [(70, 70), (1, 90), (33, 260), (129, 200), (17, 9), (0, 12), (64, 64)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name,seqs", [("one", ONE), ("draft", DRAFT), ("chunk", CHUNK)])
@pytest.mark.parametrize("heads,group,d,page", [(2, 4, 128, 16), (1, 1, 64, 32), (3, 3, 80, 16),
                                                (1, 8, 256, 64), (2, 7, 16, 128)])
def test_lengths(dtype, name, seqs, heads, group, d, page):
    s = Sequences(7, seqs, heads, group, d, page, DTYPES[dtype], amp=1.5)
    s.check(ops.paged_attention(*s.args()), what=name)


@pytest.mark.parametrize("d", range(16, 257, 16))
def test_head_sizes(d):
    s = Sequences(d, [(1, 77), (20, 45)], 2, 2, d, 32, torch.float16)
    s.check(ops.paged_attention(*s.args()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 5000])
def test_windows(dtype, window):
    s = Sequences(11, [(1, 300), (1, 5), (40, 200), (90, 90), (6, 3)], 2, 2, 64, 16, DTYPES[dtype])
    s.check(ops.paged_attention(*s.args(), window=window), window=window)
    t = Sequences(12, [(1, 300), (1, 5), (1, 130)], 2, 2, 64, 16, DTYPES[dtype])
    t.check(ops.paged_attention(*t.args(), window=window), window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 4, 40])
def test_long_axis_split(dtype, new):
    """Few rows over long sequences, whatever the caller says of the lengths."""
    s = Sequences(13, [(new, 5000), (new, 63), (new, 2049)], 1, 2, 128, 64, DTYPES[dtype])
    args = s.args()
    for max_len in (None, 5000, 1, 100000):
        s.check(ops.paged_attention(*args, max_len=max_len), what=f"max_len {max_len}")
    w = 1000
    s.check(ops.paged_attention(*args, window=w), window=w)


@pytest.mark.parametrize("new", [1, 3, 50])
@pytest.mark.parametrize("amp,scale", [(1.0, 1.0), (300.0, None), (1.0, 1e-3), (1e-20, None)])
def test_scales(new, amp, scale):
    """One key far above the others, all keys equal, and all between."""
    for dtype in ("f16", "bf16", "f32"):
        if dtype == "f16" and amp == 1e-20:
            continue
        s = Sequences(14, [(new, 90), (new, new + 1)], 2, 2, 64, 16, DTYPES[dtype], amp=amp)
        s.check(ops.paged_attention(*s.args(), scale=scale), scale=scale, what=dtype)


def test_value_scales_far_apart():
    """Tokens whose values are 2^40 times others': the large ones last, first, and hidden."""
    for where in (0, 50, 89):
        for dtype in ("bf16", "f32"):
            s = Sequences(15, [(1, 90), (60, 90)], 1, 2, 64, 16, DTYPES[dtype])
            for b in range(2):
                pg, off = divmod(s.slot(b, where), 16)
                s.vs[pg, :, off] *= 2.0 ** 40
            s.check(ops.paged_attention(*s.args()), what=f"{where} {dtype}")


@pytest.mark.parametrize("new", [1, 4, 70])
def test_not_finite_in_seen_and_hidden_places(new):
    """A NaN scale (a token that was not finite when written) makes the rows that see it NaN and
    no other row: not earlier tokens, nor rows whose window has left it behind."""
    for which in ("ks", "vs"):
        for j in (99 - new + 1, 20, 99):
            for window in (0, 30):
                s = Sequences(16, [(new, 100), (new, 80)], 2, 2, 64, 16, torch.bfloat16)
                pg, off = divmod(s.slot(0, j), 16)
                getattr(s, which)[pg, 1, off] = np.nan
                out = ops.paged_attention(*s.args(), window=window)
                s.check(out, window=window, what=f"{which} {j}")


def test_infinite_query():
    """A query with an infinity or a NaN spoils its own row only."""
    for new in (1, 40):
        s = Sequences(17, [(new, 100), (new, 60)], 2, 2, 64, 16, torch.float32)
        args = s.args()
        want = ops.paged_attention(*args)
        q = args[0].clone()
        q[0, 1, 5], q[new, 3, 0] = float("inf"), float("nan")
        got = ops.paged_attention(q, *args[1:])
        same = torch.ones(q.shape[:2], dtype=torch.bool)
        same[0, 1] = same[new, 3] = False
        assert torch.equal(got[same.cuda()], want[same.cuda()])
        assert torch.isnan(got[~same.cuda()]).all()


def test_pages_outside_the_cache():
    """A table entry that names no page hides its positions."""
    for new in (1, 30):
        s = Sequences(18, [(new, 100), (new, 80)], 2, 2, 64, 16, torch.bfloat16)
        s.table[0, 2] = s.pages
        s.table[1, 0] = -1
        s.table[1, 4] = 2 ** 31 - 1
        s.check(ops.paged_attention(*s.args()))
        s.table[:] = -1
        assert not ops.paged_attention(*s.args()).any()


def test_padded_batch_and_lengths_past_the_table():
    """Tokens past the last sequence are zeros; a length past the table's pages is cut."""
    for new in (1, 25):
        s = Sequences(19, [(new, 64), (new, 64)], 2, 2, 64, 16, torch.float16, pad_tokens=9)
        out = torch.full_like(s.q.cuda(), 3.0)
        got = ops.paged_attention(*s.args(), out=out)
        assert not got[2 * new:].any()
        s.check(got)
        q, cache, table, lens, starts = s.args()
        assert torch.equal(ops.paged_attention(q, cache, table, lens + 1000, starts), got)
        assert not ops.paged_attention(q, cache, table, lens - 1000, starts).any()


def test_strided_queries():
    """q as a slice of a projection's output, off 16 bytes too, and head-major."""
    for new in (1, 30):
        for dtype in DTYPES.values():
            s = Sequences(20, [(new, 50), (new, 90)], 2, 2, 48, 16, dtype)
            q, *rest = s.args()
            want = ops.paged_attention(q, *rest)
            for lead in (0, 8, 3):
                wide = torch.zeros((q.shape[0], lead + 4 * 48 + 16), dtype=dtype, device="cuda")
                view = wide[:, lead:lead + 4 * 48].unflatten(1, (4, 48))
                view.copy_(q)
                assert torch.equal(ops.paged_attention(view, *rest), want)
            head_major = q.transpose(0, 1).contiguous().transpose(0, 1)
            assert torch.equal(ops.paged_attention(head_major, *rest), want)


def test_same_answer_every_time():
    """Partial results are joined in a fixed order."""
    s = Sequences(21, [(1, 3000), (1, 700), (9, 2000)], 2, 4, 128, 64, torch.bfloat16)
    args = s.args()
    first = ops.paged_attention(*args)
    for _ in range(5):
        assert torch.equal(ops.paged_attention(*args), first)


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of codes."""
    heads, d, page = 8, 256, 1024
    pages = (1 << 32) // (heads * d * page) + 2
    for new in (1, 40):
        s = Sequences(22, [(new, 1500), (new, 60)], heads, 1, d, page, torch.float16)
        q, small, table, lens, starts = s.args()
        cache = ops.PagedCache.empty(pages, heads, page, d)
        top = pages - s.pages
        for big, part in zip((cache.k, cache.v, cache.k_scale, cache.v_scale),
                             (small.k, small.v, small.k_scale, small.v_scale)):
            big[top:].copy_(part)
        got = ops.paged_attention(q, cache, torch.where(table >= 0, table + top, table), lens,
                                  starts)
        assert torch.equal(got, ops.paged_attention(q, small, table, lens, starts))
        s.check(got)


def test_other_stream_and_graph():
    """Enqueued on torch's current stream; captured once and replayed with other queries, pages
    and lengths."""
    for new in (1, 6, 40):
        cases = [Sequences(30 + i, [(new, 900 - 37 * i), (new, 120 + i), (new, new)], 2, 4, 128, 32,
                           torch.bfloat16, spare_pages=3 + i) for i in range(3)]
        pages = max(c.pages for c in cases)
        width = max(c.table.shape[1] for c in cases)
        args = []
        for c in cases:
            q, small, table, lens, starts = c.args()
            cache = ops.PagedCache.empty(pages, 2, 32, 128)
            for big, part in zip((cache.k, cache.v, cache.k_scale, cache.v_scale),
                                 (small.k, small.v, small.k_scale, small.v_scale)):
                big[:c.pages].copy_(part)
            wide = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
            wide[:, :table.shape[1]] = table
            args.append((q, cache, wide, lens, starts))
        want = [ops.paged_attention(*a) for a in args]
        for c, w in zip(cases, want):
            c.check(w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = ops.paged_attention(*args[1])
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, want[1])
        q, cache, table, lens, starts = (
            ops.PagedCache(a.k.clone(), a.v.clone(), a.k_scale.clone(), a.v_scale.clone())
            if isinstance(a, ops.PagedCache) else a.clone() for a in args[0])
        ws = ops.paged_attention_workspace(q, cache, table)
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
        for a, ref in zip(args * 2, want * 2):
            q.copy_(a[0])
            for n in ("k", "v", "k_scale", "v_scale"):
                getattr(cache, n).copy_(getattr(a[1], n))
            table.copy_(a[2])
            lens.copy_(a[3])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
            assert torch.equal(ops.paged_attention(*a), ref)


def test_no_tokens():
    s = Sequences(23, [(1, 4)], 1, 1, 16, 16, torch.float32)
    q, cache, table, lens, starts = s.args()
    assert ops.paged_attention(q[:0], cache, table, lens, starts * 0).shape == (0, 1, 16)


def test_a_write_then_attention():
    """What cache_write stored is what attention reads."""
    s = Sequences(24, [(3, 40), (1, 17)], 2, 2, 64, 16, torch.float32)
    q, cache, table, lens, starts = s.args()
    r = np.random.default_rng(1)
    k = torch.from_numpy(r.standard_normal((4, 2, 64))).float()
    v = torch.from_numpy(r.standard_normal((4, 2, 64))).float()
    slots = [s.slot(0, 37), s.slot(0, 38), s.slot(0, 39), s.slot(1, 16)]
    ops.cache_write(cache, k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    s.kc, s.vc = cache.k.cpu().numpy(), cache.v.cpu().numpy()
    s.ks, s.vs = cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
    pg, off = divmod(slots[3], 16)
    assert np.allclose(s.kc[pg, :, off] * s.ks[pg, :, off][:, None], f64(k)[3], atol=0.02)
    s.check(ops.paged_attention(q, cache, table, lens, starts))
