"""Attention over the 4-bit cache where its rules change and beside memory that nothing has written:
against the 64-bit oracle, with the bounds of the other tests."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2112_13896_amd import ops
from tests.mx4_util import DTYPES, Sequences

pytestmark = pytest.mark.gpu


def garbage(s, window=0):
    """Random bytes, scales of every value among them, wherever no new token sees the cache; the
    arrays as they were, which the oracle, whose hidden weights of 0 want finite values, takes."""
    clean = [a.copy() for a in (s.kc, s.ks, s.vc, s.vs)]
    seen = np.zeros((s.pages, s.page), dtype=bool)
    for b, (new, m) in enumerate(s.seqs):
        first = max(m - new - window + 1, 0) if window else 0
        for j in range(first if new else m, m):
            seen[s.table[b, j // s.page], j % s.page] = True
    pg, off = np.nonzero(~seen)
    r = np.random.default_rng(1)
    for c, sc in ((s.kc, s.ks), (s.vc, s.vs)):
        for h in range(s.heads):
            c[pg, h, off] = r.integers(0, 16, (len(pg), c.shape[-1]))
            sc[pg, h, off] = r.integers(0, 256, (len(pg), sc.shape[-1]))
    return clean


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("new,d", [(1, 128), (7, 128), (1, 256), (7, 48), (70, 128), (70, 80)])
def test_unwritten_slots(dtype, window, new, d):
    """Slots that hold any bytes at all: behind the last token, in pages of no sequence, and before
    the first position that a window leaves."""
    s = Sequences(31, [(new, 203), (new, 75), (new, max(new, 5))], 1, 4, d, 16, DTYPES[dtype])
    clean = garbage(s, window)
    out = ops.paged_attention(*s.args(), window=window)
    s.kc, s.ks, s.vc, s.vs = clean
    s.check(out, window=window)


def test_unwritten_slots_of_a_split_axis():
    for new in (1, 5, 90):
        s = Sequences(32, [(new, 4133), (new, 2500)], 1, 4, 128, 64, torch.bfloat16)
        clean = garbage(s)
        q, cache, table, lens, starts = s.args()
        ws = ops.paged_attention_workspace(q, cache, table)
        assert ws.numel() > 0
        ws.view(torch.uint8).fill_(255)                    # what it holds does not matter either
        out = ops.paged_attention(q, cache, table, lens, starts, ws=ws)
        s.kc, s.ks, s.vc, s.vs = clean
        s.check(out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,rows", [(4, 16), (5, 32), (20, 32), (21, 128), (28, 128), (29, 128)])
def test_rows_at_the_rules_ends(dtype, new, rows):
    """16, 20, 80, 84, 112 and 116 rows of a sequence, with ends of tiles inside a token."""
    if dtype == "f32" and new in (21, 28):
        rows = 32
    s = Sequences(33, [(new, 150), (new, new), (new, 40)], 2, 4, 128, 32, DTYPES[dtype])
    plan = ops.paged_attention_plan(DTYPES[dtype], 2, 32, 128, 3 * new, 8, 3, s.table.shape[1],
                                    bits=4)
    assert plan["rows"] == rows
    s.check(ops.paged_attention(*s.args()))
    # the same total, unevenly: a sequence of most of the rows, of one token, of none
    s = Sequences(34, [(3 * new - 1, 3 * new + 9), (1, 77), (0, 30)], 2, 4, 128, 32, DTYPES[dtype])
    s.check(ops.paged_attention(*s.args()))


@pytest.mark.parametrize("new", [1, 6, 40])
@pytest.mark.parametrize("len_", [2047, 2048, 2049, 2112, 2113])
def test_axes_at_the_rules_ends(new, len_):
    """The longest whole axis, and the shortest in parts."""
    s = Sequences(35, [(new, len_), (new, 100)], 1, 4, 64, 16, torch.bfloat16)
    s.check(ops.paged_attention(*s.args(), max_len=len_), max_len=len_)
    s.check(ops.paged_attention(*s.args()))


@pytest.mark.parametrize("new", [1, 5, 30])
@pytest.mark.parametrize("past", [60, 3000])
def test_padded_batch(new, past):
    """Tokens behind the last sequence get zeros, whole axis or parts; the output before the call
    does not matter."""
    s = Sequences(36, [(new, past), (0, 9), (new, 48)], 2, 2, 64, 16, torch.float16, pad_tokens=37)
    args = s.args()
    out = torch.full(s.q.shape, float("nan"), dtype=s.q.dtype, device="cuda")
    ops.paged_attention(*args, out=out)
    s.check(out)
    assert not out[2 * new:].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 9])
def test_many_sequences_most_without_tokens(dtype, new):
    """More sequences than are added up at once, in whole axes and in parts."""
    r = np.random.default_rng(2)
    for long in (0, 2300):
        seqs = [(int(r.integers(1, new + 1)) if i % 5 == 2 or i in (0, 63, 64, 129) else 0,
                 int(r.integers(new, 90))) for i in range(133)]
        seqs[64] = (seqs[64][0], max(long, 50))
        s = Sequences(37, seqs, 1, 3, 64, 16, DTYPES[dtype])
        s.check(ops.paged_attention(*s.args()))


def test_no_sequence_has_tokens():
    """Starts of a step that was refused: all zeros."""
    for new, past in ((1, 30), (1, 4000), (60, 90), (90, 4000)):
        s = Sequences(38, [(new, past), (new, past)], 1, 4, 64, 16, torch.bfloat16)
        q, cache, table, lens, starts = s.args()
        out = torch.full_like(q, float("nan"))
        ops.paged_attention(q, cache, table.fill_(-1), lens.zero_(), starts.zero_(), out=out)
        assert not out.any()


def test_rows_past_the_widest_launch():
    """Sequences, heads and lengths whose product of workgroups passes 65,535."""
    s = Sequences(39, [(1, 1 + i % 3) for i in range(2200)], 32, 1, 16, 16, torch.float16,
                  spare_pages=1)
    s.check(ops.paged_attention(*s.args()))


def test_two_graphs_share_a_split_workspace():
    """Two recorded calls over axes in parts, with one workspace, replayed in turn."""
    graphs = []
    cases = [Sequences(40, [(1, 3100)], 2, 4, 64, 16, torch.float16),
             Sequences(41, [(1, 2900)], 2, 4, 64, 16, torch.float16)]
    args = [s.args() for s in cases]
    ws = max((ops.paged_attention_workspace(a[0], a[1], a[2]) for a in args),
             key=lambda w: w.numel())
    assert ws.numel() > 0
    for a in args:
        out = torch.empty_like(a[0])
        ops.paged_attention(*a, ws=ws, out=out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.paged_attention(*a, ws=ws, out=out)
        graphs.append((g, out))
    for _ in range(3):
        for _, out in graphs:
            out.zero_()
        for g, _ in graphs:
            g.replay()
        for s, (_, out) in zip(cases, graphs):
            s.check(out)
