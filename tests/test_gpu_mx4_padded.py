"""Attention over the 4-bit cache in padded batches: most entries of the table bring no token."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import ops
from tests.mx4_util import DTYPES, Sequences

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 7, 30])
def test_few_sequences_of_a_large_table(dtype, new):
    """Three sequences with tokens, first, between and last of 150 entries, over axes in parts."""
    seqs = [(0, 20)] * 150
    seqs[0], seqs[70], seqs[149] = (new, 4133), (1, 63), (new, 2500)
    s = Sequences(61, seqs, 2, 4, 128, 64, DTYPES[dtype])
    q, cache, table, lens, starts = s.args()
    plan = ops.paged_attention_plan(DTYPES[dtype], 2, 64, 128, len(q), 8, 150, table.shape[1],
                                    bits=4)
    assert new == 30 or plan["parts"] > 1
    ws = ops.paged_attention_workspace(q, cache, table)
    ws.fill_(255)                                          # what it holds does not matter
    out = torch.full_like(q, float("nan"))
    ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
    s.check(out)


def test_a_padded_batch_recorded():
    """A table of 40 entries of which other ones bring the tokens at each replay, the last of them
    padding."""
    s = Sequences(62, [(1, 3000), (1, 2200), (1, 90)] + [(0, 5)] * 37, 1, 4, 64, 64, torch.bfloat16)
    q, cache, table, lens, starts = s.args()
    out = torch.empty_like(q)
    ws = ops.paged_attention_workspace(q, cache, table)
    assert ws.numel() > 0
    ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.paged_attention(q, cache, table, lens, starts, ws=ws, out=out)
    for new in ((1, 1, 1), (0, 1, 0), (2, 0, 1), (0, 0, 0), (0, 0, 3)):
        begins = [0]
        for n in (*new, *[0] * 37):
            begins.append(begins[-1] + n)
        starts.copy_(torch.tensor(begins, dtype=torch.int32))
        graph.replay()
        got = out.clone()
        assert torch.equal(got, ops.paged_attention(q, cache, table, lens, starts))
        s.seqs = [(n, m) for n, (_, m) in zip((*new, *[0] * 37), s.seqs)]
        s.starts = starts.cpu().numpy()
        s.check(got)
        assert not got[begins[-1]:].any()
