"""Paged attention over the 4-bit cache against the 64-bit oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2112_13896_amd import ops
from tests.mx4_util import DTYPES, Sequences, f64

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


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", range(16, 257, 16))
def test_head_sizes(dtype, d):
    for seqs in ([(1, 77), (2, 45)], [(1, 77), (90, 95)]):
        s = Sequences(d, seqs, 2, 2, d, 32, DTYPES[dtype])
        s.check(ops.paged_attention(*s.args()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 5000])
def test_windows(dtype, window):
    for seqs in ([(1, 300), (1, 5), (40, 200), (90, 90), (6, 3)], [(1, 300), (1, 5), (1, 130)]):
        s = Sequences(11, seqs, 2, 2, 64, 16, DTYPES[dtype])
        s.check(ops.paged_attention(*s.args(), window=window), window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 4, 40, 90])
def test_long_axis_split(dtype, new):
    """Few rows over long sequences, whatever the caller says of the lengths."""
    s = Sequences(13, [(new, 5000), (new, 63), (new, 2049)], 1, 2, 128, 64, DTYPES[dtype])
    args = s.args()
    for max_len in (None, 5000, 1, 100000):
        s.check(ops.paged_attention(*args, max_len=max_len), what=f"max_len {max_len}",
                max_len=max_len)
    w = 1000
    s.check(ops.paged_attention(*args, window=w), window=w)


@pytest.mark.parametrize("new", [1, 3, 50, 80])
@pytest.mark.parametrize("amp,scale", [(1.0, 1.0), (300.0, None), (1.0, 1e-3), (1e-20, None)])
def test_scales(new, amp, scale):
    """One key far above the others, all keys equal, and all between."""
    for dtype in ("f16", "bf16", "f32"):
        if dtype == "f16" and amp == 1e-20:
            continue
        s = Sequences(14, [(new, 90), (new, new + 1)], 2, 2, 64, 16, DTYPES[dtype], amp=amp)
        s.check(ops.paged_attention(*s.args(), scale=scale), scale=scale, what=dtype)


@pytest.mark.parametrize("by", [-50, 40])
def test_scales_far_apart(by):
    """Tokens whose keys or values are far larger or smaller than others', whole rows and single
    groups; the odd ones last, first, between, and hidden from some rows."""
    for which in "kv":
        for where in (0, 50, 89):
            for dtype in ("bf16", "f32"):
                s = Sequences(15, [(1, 90), (70, 90)], 1, 2, 64, 16, DTYPES[dtype])
                for b in range(2):
                    pg, off = divmod(s.slot(b, where), 16)
                    sc = getattr(s, which + "s")
                    if which == "k":
                        sc[pg, :, off] = np.clip(sc[pg, :, off].astype(int) + min(by, 8), 67, 187)
                    elif b:
                        sc[pg, :, off, 1] = np.clip(sc[pg, :, off, 1].astype(int) + by, 67, 187)
                    else:
                        sc[pg, :, off] = np.clip(sc[pg, :, off].astype(int) + by, 67, 187)
                s.check(ops.paged_attention(*s.args()), what=f"{which} {where} {dtype}")


def test_values_at_both_ends_of_the_scales():
    """All values at the largest scale, and all at the smallest: sums neither pass 32-bit floats
    nor vanish."""
    for byte in (67, 187):
        for dtype in ("bf16", "f32"):
            s = Sequences(19, [(1, 90), (70, 150)], 1, 2, 64, 16, DTYPES[dtype])
            s.vs[s.vs != 255] = byte
            s.check(ops.paged_attention(*s.args()), what=f"{byte} {dtype}")


@pytest.mark.parametrize("new", [1, 4, 70])
def test_not_finite_in_seen_and_hidden_places(new):
    """A token that was not finite when written makes the rows that see it NaN and no other row:
    not earlier tokens, nor rows whose window has left it behind."""
    for which in "kv":
        for j in (99 - new + 1, 20, 99):
            for window in (0, 30):
                s = Sequences(16, [(new, 100), (new, 80)], 2, 2, 64, 16, torch.bfloat16)
                pg, off = divmod(s.slot(0, j), 16)
                s.spoil(which, pg, 1, off)
                out = ops.paged_attention(*s.args(), window=window)
                s.check(out, window=window, what=f"{which} {j}")


def test_infinite_query():
    """A query with an infinity or a NaN spoils its own row only."""
    for dtype in (torch.float32, torch.bfloat16):
        for new in (1, 40):
            s = Sequences(17, [(new, 100), (new, 60)], 2, 2, 64, 16, dtype)
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
    for new in (1, 30, 70):
        s = Sequences(18, [(new, 100), (new, 80)], 2, 2, 64, 16, torch.bfloat16)
        s.table[0, 2] = s.pages
        s.table[1, 0] = -1
        s.table[1, 4] = 2 ** 31 - 1
        s.check(ops.paged_attention(*s.args()))
        s.table[:] = -1
        assert not ops.paged_attention(*s.args()).any()


def test_padded_batch_and_lengths_past_the_table():
    """Tokens past the last sequence get zeros; lengths past the table are cut to it."""
    for new in (1, 30):
        s = Sequences(20, [(new, 60), (new, 48)], 2, 2, 64, 16, torch.float16, pad_tokens=5)
        q, cache, table, lens, starts = s.args()
        out = ops.paged_attention(q, cache, table, lens, starts)
        s.check(out)
        assert not out[2 * new:].any()
        long = lens.clone()
        long[0] = 10 ** 9
        s.lens[0] = 64                                     # four pages of 16: what the table holds
        s.seqs = [(new, 64), (new, 48)]
        s.check(ops.paged_attention(q, cache, table, long, starts))


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_alignment(dtype):
    """Queries inside a wider tensor, and on addresses that are no multiple of 16 bytes."""
    for new in (1, 70):
        s = Sequences(21, [(new, 100), (new, 70)], 2, 2, 80, 16, DTYPES[dtype])
        q, *rest = s.args()
        want = ops.paged_attention(q, *rest)
        wide = torch.full((2 * new, 11, 80), 7.0, dtype=q.dtype, device="cuda")
        wide[:, 3:7] = q
        assert torch.equal(ops.paged_attention(wide[:, 3:7], *rest), want)
        flat = torch.zeros(2 * new * 4 * 83 + 1, dtype=q.dtype, device="cuda")
        odd = flat[1:].view(2 * new, 4, 83)[:, :, 2:82]
        odd.copy_(q)
        assert torch.equal(ops.paged_attention(odd, *rest), want)


def test_same_bits_again_and_on_another_stream():
    s = Sequences(22, [(1, 3000), (3, 200), (1, 2500)], 2, 4, 128, 64, torch.bfloat16)
    args = s.args()
    want = ops.paged_attention(*args)
    s.check(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [ops.paged_attention(*args) for _ in range(3)]
    side.synchronize()
    for g in got:
        assert torch.equal(g, want)


def test_captured_and_replayed():
    """Recorded once; lengths, pages and queries change between the replays."""
    s = Sequences(23, [(1, 2900), (1, 100)], 2, 4, 128, 64, torch.bfloat16)
    q, cache, table, lens, starts = s.args()
    out = torch.empty_like(q)
    ws = ops.paged_attention_workspace(q, cache, table)
    ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
    for n0, n1 in ((2900, 100), (7, 64), (2048, 1)):
        lens.copy_(torch.tensor([n0, n1], dtype=torch.int32))
        q.copy_(torch.randn(q.shape, device="cuda"))
        graph.replay()
        got = out.clone()
        assert torch.equal(got, ops.paged_attention(q, cache, table, lens, starts))
        s.q, s.lens = q.cpu(), np.array([n0, n1], np.int32)
        s.seqs = [(1, n0), (1, n1)]
        s.check(got)


def test_offsets_past_32_bits():
    """Pages at the end of a cache of more than 2^32 bytes of keys."""
    heads, page, d = 8, 1024, 256
    pages = 2 ** 32 // (heads * page * d // 2) + 3
    s = Sequences(24, [(1, 40), (20, 30)], heads, 1, d, page, torch.bfloat16, spare_pages=0)
    small = s.cache()
    big = ops.PagedCache4.empty(pages, heads, page, d)
    far = torch.tensor([pages - 1, pages - 2], device="cuda")
    near = torch.from_numpy(s.table[:, 0].astype(np.int64)).cuda()
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(big, name)[far] = getattr(small, name)[near]
    q, _, _, lens, starts = s.args()
    table = far.int()[:, None].contiguous()
    s.check(ops.paged_attention(q, big, table, lens, starts))
    k, v = (torch.randn((2, heads, d), device="cuda") for _ in "kv")
    slots = torch.tensor([pages * page - 1, (pages - 1) * page - 5], device="cuda")
    ops.cache_write(big, k, v, slots)
    other = ops.PagedCache4.empty(1, heads, 16, d)
    two = torch.tensor([0, 1], device="cuda")
    ops.cache_write(other, k, v, two)
    for a, b in zip(ops.cache_read(big, slots, torch.float32),
                    ops.cache_read(other, two, torch.float32)):
        assert torch.equal(a, b)


def test_no_tokens():
    s = Sequences(25, [(1, 20)], 2, 2, 32, 16, torch.float16)
    q, cache, table, lens, starts = s.args()
    out = ops.paged_attention(q[:0], cache, table, lens, starts)
    assert out.shape == (0, 4, 32)
    assert f64(out).size == 0
