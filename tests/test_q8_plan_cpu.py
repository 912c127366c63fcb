"""Host bookkeeping of the 8-bit attention layer: pages and steps."""
from __future__ import annotations

import pytest

from paper_2112_13896_amd.attention import PagePool, Sequence, Step


def test_pool():
    pool = PagePool(4, 16)
    a, b = Sequence(), Sequence()
    pool.extend(a, 16)
    assert len(a.pages) == 1 and len(pool) == 3
    pool.extend(a, 1)
    pool.extend(b, 0)
    assert len(a.pages) == 2 and a.length == 17 and b.pages == []
    with pytest.raises(RuntimeError):
        pool.extend(b, 33)
    assert b.length == 0 and len(pool) == 2
    pool.extend(b, 32)
    assert len(pool) == 0 and len(set(a.pages + b.pages)) == 4
    pool.extend(a, 15)                                       # fits the page it has
    pool.release(a)
    assert len(pool) == 2 and a.length == 0
    with pytest.raises(ValueError):
        pool.extend(a, -1)


def test_step():
    a, b, c = Sequence([5, 2], 20), Sequence([], 0), Sequence([7], 16)
    s = Step.of([a, b, c], [3, 0, 16], 16, device="cpu", width=4)
    assert s.table.tolist() == [[5, 2, -1, -1], [-1] * 4, [7, -1, -1, -1]]
    assert s.lens.tolist() == [20, 0, 16] and s.starts.tolist() == [0, 3, 3, 19]
    assert s.slots.tolist() == [2 * 16 + 1, 2 * 16 + 2, 2 * 16 + 3] + list(range(112, 128))
    assert s.max_len == 20
    for seqs, new in (([], []), ([a], [1, 2]), ([a], [21]), ([a], [-1]),
                      ([Sequence([1], 17)], [1])):
        with pytest.raises(ValueError):
            Step.of(seqs, new, 16, device="cpu")
