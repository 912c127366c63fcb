"""Steps planned on the GPU against a pool of pages on the host."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as o4
from paper_2112_13896_amd import ops
from paper_2112_13896_amd.attention import PagePool, Sequence, Step

pytestmark = pytest.mark.gpu

I32 = torch.int32


def _gpu(a):
    return torch.tensor(a, dtype=I32, device="cuda")


class Both:
    """The same calls on the GPU's pool and on the host's."""

    def __init__(self, sequences, width, pages, page):
        self.gpu = ops.DevicePool.empty(sequences, width, pages, page)
        self.host = o4.Pool(sequences, width, pages, page)

    def plan(self, seqs, new, tokens, width=None, status=0):
        got = ops.plan_step(self.gpu, _gpu(seqs), _gpu(new), tokens, width)
        want = self.host.plan(seqs, new, tokens, width)
        for g, w, name in zip(got, want, ("table", "lens", "starts", "slots", "positions",
                                          "status")):
            assert np.array_equal(g.cpu().numpy(), w), (name, g.cpu().numpy(), w)
        assert int(got[5][0]) == status
        self.same()
        return got

    def truncate(self, seqs, lens=None):
        ops.pool_truncate(self.gpu, _gpu(seqs), None if lens is None else _gpu(lens))
        self.host.truncate(seqs, lens)
        self.same()

    def same(self):
        h = self.host
        assert self.gpu.lengths.tolist() == h.lengths
        n = int(self.gpu.count)
        assert self.gpu.free[:n].tolist() == h.free
        table = self.gpu.table.cpu().numpy()
        for s, held in enumerate(h.held):
            assert table[s, :len(held)].tolist() == held
        assert bool((self.gpu.marks == 2 ** 31 - 1).all())


def test_a_life_of_sequences():
    b = Both(6, 8, 30, 16)
    b.plan([0, 3], [17, 1], 20)
    b.plan([3, 1, 0], [1, 40, 15], 56)
    b.plan([5], [0], 0)
    b.truncate([0, 1], [16, 33])
    b.plan([1, 0, 2, -1], [5, 1, 16, 9], 40)
    b.truncate([1])
    b.truncate([0, 2, 3, 4, 5])
    assert len(b.host.free) == 30


@pytest.mark.parametrize("seed", range(6))
def test_random_steps(seed):
    r = np.random.default_rng(seed)
    sequences = [5, 40, 1500, 2500, 3, 300][seed]
    page = [16, 32, 64, 16, 1024, 128][seed]
    width = [4, 9, 7, 30, 2, 5][seed]
    b = Both(sequences, width, sequences * width * 2 // 3 + 2, page)
    for _ in range(6):
        n = int(r.integers(1, sequences + 1))
        seqs = r.permutation(sequences)[:n]
        room = width * page - np.array(b.host.lengths)[seqs]
        new = np.minimum(r.integers(0, page * 2, n), room)
        seqs = np.where(r.random(n) < 0.1, -1, seqs)
        total = int(new[seqs >= 0].sum())
        need = sum(-(-(b.host.lengths[s] + m) // page) - len(b.host.held[s])
                   for s, m in zip(seqs, new) if s >= 0)
        fits = need <= len(b.host.free)
        b.plan(seqs.tolist(), new.tolist(), total + int(r.integers(0, 5)),
               width if r.random() < 0.5 else width + 3, status=0 if fits else 3)
        cut = r.permutation(sequences)[:int(r.integers(1, sequences + 1))]
        to = [int(r.integers(0, b.host.lengths[s] + 1)) for s in cut]
        if r.random() < 0.7:
            b.truncate(cut.tolist(), to)
        else:
            b.truncate(cut[:3].tolist())


def test_wrong_entries_change_nothing():
    b = Both(4, 4, 9, 16)
    b.plan([0, 1], [20, 3], 23)
    for seqs, new, tokens, status in (([0, 4], [1, 1], 9, 1), ([-2], [1], 9, 1),
                                      ([2, 2], [1, 1], 9, 1),
                                      ([1, 0, 1], [0, 0, 0], 9, 1), ([0], [-1], 9, 1),
                                      ([0], [45], 99, 1), ([0], [2 ** 31 - 1], 99, 1),
                                      ([0, 1], [3, 4], 6, 2), ([2, 3], [64, 64], 200, 3)):
        b.plan(seqs, new, tokens, status=status)
    b.plan([0], [13], 20, width=2, status=1)                  # 33 positions, 2 pages of 16
    b.plan([0], [12], 20, width=2)


def test_truncate_leaves_wrong_entries_out():
    b = Both(4, 4, 12, 16)
    b.plan([0, 1, 2], [50, 17, 3], 70)
    b.truncate([4, -1, -7, 0, 0, 1], [0, 0, 0, 33, 1, 18])    # unknown, twice, longer than it is
    b.truncate([0, 1], [-1, 17])
    b.truncate([3])


def test_a_step_taken_back_leaves_the_stack():
    b = Both(70, 20, 900, 16)
    b.plan(list(range(70)), [int(n) for n in np.random.default_rng(3).integers(0, 100, 70)], 7000)
    before, stack, count = b.gpu.lengths.clone(), b.gpu.free.clone(), b.gpu.count.clone()
    seqs = _gpu(list(range(69, -1, -1)))
    step = ops.plan_step(b.gpu, seqs, _gpu([37] * 70), 70 * 37)
    assert step[5].tolist() == [0, 0]
    ops.pool_truncate(b.gpu, seqs, before[seqs.long()].contiguous())
    for a, c in ((b.gpu.lengths, before), (b.gpu.free, stack), (b.gpu.count, count)):
        assert torch.equal(a, c)
    b.same()


def test_the_hosts_pool_and_step_agree():
    """PagePool and Step.of give the same pages, tables and slots."""
    pool, seqs = PagePool(40, 16), [Sequence() for _ in range(3)]
    dev = ops.DevicePool.empty(3, 9, 40, 16)
    for new in ([30, 1, 5], [1, 1, 1], [0, 16, 40]):
        for s, n in zip(seqs, new):
            pool.extend(s, n)
        want = Step.of(seqs, new, 16, width=9)
        table, lens, starts, slots, _, status = ops.plan_step(dev, _gpu([0, 1, 2]), _gpu(new),
                                                              sum(new))
        assert status.tolist() == [0, 0]
        for a, c in ((table, want.table), (lens, want.lens), (starts, want.starts),
                     (slots, want.slots)):
            assert torch.equal(a, c)


def test_captured_and_replayed():
    """A recorded step advances the pool at each replay, eager work between them."""
    b = Both(5, 6, 30, 16)
    b.plan([0, 1, 2, 3, 4], [3, 14, 15, 16, 40], 88)
    seqs, new = _gpu([4, 2, 0, -1]), _gpu([1, 1, 1, 0])
    out = ops.plan_step(b.gpu, seqs, new, 4)
    ws = ops.plan_step_workspace(4)
    ops.pool_truncate(b.gpu, seqs[:3], _gpu([40, 15, 3]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.plan_step(b.gpu, seqs, new, 4, ws=ws, out=out)
    for i in range(20):
        graph.replay()
        want = b.host.plan([4, 2, 0, -1], [1, 1, 1, 0], 4)
        for g, w in zip(out, want):
            assert np.array_equal(g.cpu().numpy(), w), i
        b.same()
        if i == 9:
            b.truncate([2], [1])


def test_one_sequence_many_pages_and_many_sequences():
    b = Both(1, 3000, 3000, 16)
    b.plan([0], [47990], 48000)
    b.plan([0], [11], 11, status=1)
    b.plan([0], [10], 11)
    b.truncate([0], [17])
    b.truncate([0])
