"""Paged attention over values next to nothing: tokens whose value scale is far below the others',
or all of them, against the 64-bit oracle."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, Sequences

pytestmark = pytest.mark.gpu

NEW = [1, 3, 70]                                             # one token, a few, many rows


def _scale_values(s, where, factor):
    for b, (_, m) in enumerate(s.seqs):
        for j in range(m):
            if where(j, m):
                pg, off = divmod(s.slot(b, j), s.page)
                s.vs[pg, :, off] *= factor


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("d,length", [(64, 300), (128, 900), (32, 6000)])
@pytest.mark.parametrize("where", ["first", "last", "all but one", "every other"])
def test_ordinary_tokens_among_small_ones(dtype, new, d, length, where):
    """Values of 1e-36 or so beside ordinary ones: whole steps of the kernels and whole parts of a
    split axis, before and after them."""
    tiny = {"first": lambda j, m: j < m - 80, "last": lambda j, m: 10 <= j,
            "all but one": lambda j, m: j != m // 2, "every other": lambda j, m: j % 2}[where]
    s = Sequences(d + new, [(new, length), (new, 100)], 1, 2, d, 32, DTYPES[dtype])
    _scale_values(s, tiny, 5e-35)
    s.check(ops.paged_attention(*s.args()), what=where)
    s.check(ops.paged_attention(*s.args(), window=90), window=90, what=where)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -80, 2.0 ** -100, 2.0 ** -107, 2.0 ** 110])
def test_all_values_of_one_size(dtype, new, scale):
    for d, length in ((64, 300), (32, 6000)):
        s = Sequences(d + new, [(new, length), (new, 100)], 1, 2, d, 32, DTYPES[dtype])
        _scale_values(s, lambda j, m: True, scale)
        if dtype == "f16" and scale > 1:                     # past the type's largest number
            continue
        s.check(ops.paged_attention(*s.args()), what=f"{scale}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", NEW)
@pytest.mark.parametrize("keys", [20.0, 60.0, 200.0])
def test_a_small_value_that_rules_its_row(dtype, new, keys):
    """A few keys far larger than the others, so that they rule some rows and are nothing to
    others, with values next to nothing."""
    s = Sequences(int(keys) + new, [(new, 500), (new, 90)], 2, 2, 64, 32, DTYPES[dtype])
    for b, j in ((0, 0), (0, 130), (0, 420), (1, 3)):
        pg, off = divmod(s.slot(b, j), s.page)
        s.ks[pg, :, off] *= keys
        s.vs[pg, :, off] *= 1e-33
    s.check(ops.paged_attention(*s.args()))


@pytest.mark.parametrize("new", NEW)
def test_zeros_and_scales_below_normal_numbers(new):
    """Rows of scale 0 (their codes are 0) and scales that have no reciprocal, before others."""
    for dtype in (torch.bfloat16, torch.float32):
        for length in (300, 6000):
            s = Sequences(40 + new, [(new, length)], 1, 2, 64, 32, dtype)
            for j in range(length - 75):
                pg, off = divmod(s.slot(0, j), s.page)
                if j % 3 == 0:
                    s.vs[pg, :, off], s.vc[pg, :, off] = 0.0, 0
                else:
                    s.vs[pg, :, off] = 2.0 ** -149 if j % 3 == 1 else 2.0 ** -130
            s.check(ops.paged_attention(*s.args()))
