"""Windows over an axis that is split: results, and nothing written past the workspace that was
asked for.  The sizes are those where the window's axis has more parts than the whole one."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, Sequences

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


def _run(s, args, window, max_len, room_len=None):
    """paged_attention with a workspace of just the size asked for, guard bytes behind it."""
    need = ops.paged_attention_workspace(*args[:3], max_len=room_len or max_len).numel()
    buf = torch.full((need + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
    got = ops.paged_attention(*args, window=window, max_len=max_len, ws=buf[:need])
    torch.cuda.synchronize()
    assert bool((buf[need:] == 0x5A).all())
    s.check(got, window=window, what=f"window {window} max_len {max_len}")
    assert torch.equal(ops.paged_attention(*args, window=window, max_len=max_len), got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,window,length", [(1, 1728, 1800), (1, 1728, 2000), (1, 4800, 5000),
                                               (3, 7872, 8191), (70, 4800, 5000)])
def test_one_sequence(dtype, new, window, length):
    s = Sequences(window + new, [(new, length)], 1, 2, 64, 64, DTYPES[dtype])
    args = s.args()
    plan = ops.paged_attention_plan(DTYPES[dtype], 1, 64, 64, new, 2, 1, -(-length // 64), length,
                                    window)
    whole = ops.paged_attention_plan(DTYPES[dtype], 1, 64, 64, new, 2, 1, -(-length // 64), length)
    assert plan["parts"] > whole["parts"]
    _run(s, args, window, length)
    _run(s, args, 0, length)


@pytest.mark.parametrize("batch,window,length", [(42, 2048, 2496), (22, 4096, 4225)])
def test_decoding_batch(batch, window, length):
    s = Sequences(batch, [(1, length - 7 * i) for i in range(batch)], 8, 1, 32, 64, torch.bfloat16)
    args = s.args()
    sizes = (torch.bfloat16, 8, 64, 32, batch, 8, batch, -(-length // 64), length)
    assert ops.paged_attention_plan(*sizes, window)["parts"] > ops.paged_attention_plan(*sizes)["parts"]
    _run(s, args, window, length)


@pytest.mark.parametrize("new", [1, 70])
def test_a_workspace_of_the_longest_step(new):
    """What serves the longest step serves every shorter one."""
    s = Sequences(8, [(new, 4100)], 1, 2, 32, 64, torch.float16)
    args = s.args()
    for max_len in (5000, 4864, 4200, 4100):
        for window in (0, 4032):
            _run(s, args, window, max_len, room_len=5000)
