"""The layer's recorded steps with workspaces that they share and that the kernels do pass data
through: plans of two launches, key axes in parts."""
from __future__ import annotations

import torch
import pytest

from paper_2112_13896_amd import ops
from paper_2112_13896_amd.attention import AttentionLayer, Step
from tests.test_gpu_mx4_layer import D, HEADS, PAGE, _gpu, _weights, _x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
def test_two_recorded_steps_in_turn(bits):
    """Plans of 66,000 cells, which two launches write, and axes of up to 4,800 positions in parts:
    two graphs over one pool and one cache, replayed in turn and alternately with eager steps."""
    dt, width, longest = torch.bfloat16, 16500, 4800
    layer = AttentionLayer(*_weights(31), HEADS, D, dtype=dt, rotary=ops.Rotary.make(D))
    pages = 1100
    cache = layer.make_cache(pages, PAGE, bits)
    pool = ops.DevicePool.empty(8, width, pages, PAGE)
    lengths = [4500, 2300, 64, 1500, 4000, 3100, 1, 90]
    for s, n in enumerate(lengths):
        step = Step.plan(pool, _gpu([s]), _gpu([n]), n, longest)
        assert step.status.tolist() == [0, 0]
        layer.forward(_x(40 + s, n, dt), cache, step)
    ids = [_gpu([0, 3, 2, 1]), _gpu([7, 5, 4, 6])]
    back = [_gpu([lengths[int(i)] for i in s.tolist()]) for s in ids]
    new = _gpu([1] * 4)
    x = [_x(50, 4, dt), _x(51, 4, dt)]
    first = Step.plan(pool, ids[0], new, 4, longest)
    buffers = layer.make_buffers(4, cache, first)
    ws = ops.plan_step_workspace(4)
    assert buffers["ws_att"].numel() > 0 and 4 * width > 32768
    layer.forward(x[0], cache, first, buffers)
    ops.pool_truncate(pool, ids[0], back[0])
    graphs, want = [], []
    for i in range(2):
        b = {k: v if k.startswith("ws") else v.clone() for k, v in buffers.items()}
        step = Step.plan(pool, ids[i], new, 4, longest)
        want.append(layer.forward(x[i], cache, step).clone())
        tables = step.table.clone()
        ops.pool_truncate(pool, ids[i], back[i])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            Step.plan(pool, ids[i], new, 4, longest, ws=ws, into=step)
            y = layer.forward(x[i], cache, step, b)
            ops.pool_truncate(pool, ids[i], back[i])
        graphs.append((g, y, step, tables, b))             # (what a graph writes stays alive)
    for turn in range(4):
        for i in (0, 1) if turn % 2 else (1, 0):
            ws.fill_(255)                                  # nothing is kept from one to the next
            buffers["ws_att"].fill_(255)
            graphs[i][1].zero_()
            graphs[i][0].replay()
            assert torch.equal(graphs[i][1], want[i]), (turn, i)
            assert torch.equal(graphs[i][2].table, graphs[i][3])
            assert graphs[i][2].status.tolist() == [0, 0]
        for g, *_ in graphs:
            g.replay()
        for i in range(2):
            assert torch.equal(graphs[i][1], want[i]), turn
    assert pool.lengths.tolist() == lengths
