"""What step plans refuse, asked through the Python calls: every refusal is before the first HIP
call."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import _lib, ops
from paper_2112_13896_amd.attention import Sequence, Step
from tests.test_q8_devices_cpu import at

I32 = torch.int32
MOST = 1 << 20                                             # entries of a step


@pytest.fixture
def stream(monkeypatch):
    monkeypatch.setattr(ops, "_current_gpu", lambda: 0)
    monkeypatch.setattr(ops, "_current_stream", lambda gpu: 0)


def _pool():
    return ops.DevicePool(at(0, 4, 3, dtype=I32), at(0, 4, dtype=I32), at(0, 9, dtype=I32),
                          at(0, 1, dtype=I32), 16)


@pytest.mark.parametrize("own", ["ws", "both", "neither"])
def test_a_step_of_too_many_entries(stream, own):
    """The library's refusal, whoever brings the workspace and the results."""
    n = MOST + 1
    seqs = at(0, n, dtype=I32)
    ws = None if own == "neither" else at(0, 256, dtype=torch.uint8)
    out = None
    if own == "both":
        out = (at(0, n, 1, dtype=I32), at(0, n, dtype=I32), at(0, n + 1, dtype=I32),
               at(0, 5, dtype=torch.int64), at(0, 5, dtype=I32), at(0, 2, dtype=I32))
    with pytest.raises(_lib.CSError, match="cs_plan_step"):
        ops.plan_step(_pool(), seqs, seqs, 5, 1, ws=ws, out=out)
    with pytest.raises(_lib.CSError, match="cs_pool_truncate"):
        ops.pool_truncate(_pool(), seqs)


def test_into_a_step_of_the_hosts(stream):
    """It has no status to write."""
    seqs = at(0, 1, dtype=I32)
    host = Step.of([Sequence([0], 3)], [2], 16, device="cpu", width=3)
    with pytest.raises(ValueError, match="into"):
        Step.plan(_pool(), seqs, seqs, 2, 16, into=host)
    host.positions, host.status = None, at(0, 2, dtype=I32)
    with pytest.raises(ValueError, match="into"):
        Step.plan(_pool(), seqs, seqs, 2, 16, into=host)
