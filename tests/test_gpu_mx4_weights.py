"""Attention over the 4-bit cache where the weights' own rounding shows: values that all but cancel.
Against the 64-bit oracle, with the bounds of the other tests, whose output rounding is then small."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as o4
from paper_2112_13896_amd import ops
from tests.mx4_util import DTYPES, Sequences, bound_attention, f64

pytestmark = pytest.mark.gpu


def cancelling(seed, seqs, d, page, dtype):
    """Two visible keys of nearly equal weight at a time, with values of 6 and of -6."""
    s = Sequences(seed, seqs, 2, 4, d, page, dtype, amp=0.05)
    for b, (_, m) in enumerate(seqs):
        for j in range(m):
            pg, off = divmod(s.slot(b, j), page)
            s.vc[pg, :, off, :d] = 15 if j % 2 else 7
            s.vs[pg, :, off] = 127
    return s


def off_by(s, out, window):
    """The largest error of the outputs, of its bound with weights of 16 bits (fp32: 24)."""
    k, v = s.dense()
    *ref, mass = o4.attention(f64(s.q), k, v, s.lens, s.starts, float(np.float32(s.d ** -0.5)),
                              window)
    tol = bound_attention(*ref, mass, int(s.lens.max()), s.d, s.dtype)
    return float((np.abs(f64(out) - ref[0]) / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 5, 40])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 64), (96, 64), (128, 32), (128, 64), (192, 64),
                                    (192, 16), (256, 64)])
def test_weights_keep_their_bits_however_many_rows_there_are(dtype, new, d, page):
    s = cancelling(51, [(new, 90), (new, 41)], d, page, DTYPES[dtype])
    assert off_by(s, ops.paged_attention(*s.args(), window=2), 2) <= 1


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_token_beside_a_prompt(dtype):
    """Decoding sequences whose batch a prompt shares: their weights have the bits that they have
    in a batch of their own."""
    for seqs in ([(1, 70), (1, 33), (1, 2)], [(1, 70), (1, 33), (200, 260)]):
        s = cancelling(52, seqs, 128, 64, DTYPES[dtype])
        assert off_by(s, ops.paged_attention(*s.args(), window=2), 2) <= 1


def test_tokens_far_apart_in_weight():
    """Weights over many keys, from 1 down to 2^-12 or so: sums that all but cancel keep the bits of
    the small ones too."""
    for dtype in DTYPES.values():
        for new in (1, 40):
            s = cancelling(53, [(new, 300), (new, 177)], 64, 64, dtype)
            s.q = (s.q.float() * 40).to(dtype)
            assert off_by(s, ops.paged_attention(*s.args()), 0) <= 1
