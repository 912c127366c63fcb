"""Numbers past 32 bits at the 8-bit operators' Python wrappers: sizes that the C interface cannot
take are refused, windows and lengths that only mean "all of it" are taken as that."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import ops
from tests.test_q8_devices_cpu import OnGpu, at, calls, rec  # noqa: F401  (rec: fixture)

BIG = 2 ** 32 + 16


def huge(shape, dtype):
    """A tensor of this shape without memory."""
    return torch.Tensor._make_subclass(OnGpu, torch.empty(shape, dtype=dtype, device="meta"))


@pytest.mark.parametrize("more", [2 ** 31, 2 ** 32, 2 ** 32 + 4, 10 ** 12, 2 ** 63 - 1])
def test_windows_and_lengths(rec, more):  # noqa: F811
    f, tensors = calls(0)["paged_attention"]
    tensors = {k: v for k, v in tensors.items() if k not in ("ws", "out")}
    tensors["ws"] = at(0, 64, dtype=torch.uint8)
    ops.paged_attention(**tensors, window=more, max_len=more)
    (_, args), = rec.calls
    max_len, window = args[12], args[14]
    assert max_len == window == 2 ** 31 - 1


def test_plan():
    sizes = (torch.bfloat16, 8, 64, 128, 3, 32, 3, 64)
    assert ops.paged_attention_plan(*sizes, max_len=2 ** 32 + 4, window=2 ** 32 + 4) == \
        ops.paged_attention_plan(*sizes)


def test_sizes(rec):  # noqa: F811
    i8, i32 = torch.int8, torch.int32
    with pytest.raises(ValueError):
        ops.quantise_rows(huge((1, BIG), torch.float16), q=huge((1, BIG), i8), scale=at(0, 1))
    with pytest.raises(ValueError):
        ops.linear_q8(at(0, 4, 32, dtype=i8), huge((BIG, 32), i8), huge((BIG,), torch.float32),
                      sx=at(0, 4), ws=at(0, 64, dtype=torch.uint8), out=huge((4, BIG), torch.float32))
    _, t = calls(0)["paged_attention"]
    with pytest.raises(ValueError):
        ops.paged_attention(**{**t, "table": huge((2, BIG), i32)})
    with pytest.raises(ValueError):
        ops.paged_attention_workspace(huge((BIG, 4, 32), torch.float32), t["cache"], t["table"])
    assert not rec.calls
