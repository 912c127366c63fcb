"""Attention over the 4-bit cache in padded batches, planned on the host: entries without tokens are
no sequences."""
import ctypes

import pytest
import torch

from paper_2112_13896_amd import _lib, ops
from paper_2112_13896_amd._lib import CS_BF16, CS_F32, CS_OK

P = 0x100000            # an aligned address that must never be dereferenced


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("group,d", [(1, 64), (4, 128), (16, 128), (100, 64), (4, 256)])
@pytest.mark.parametrize("tokens", [1, 3, 5, 40])
def test_entries_without_tokens_take_no_parts(dtype, group, d, tokens):
    """As many entries as tokens, or a table of any more: the same rows, parts and workgroups."""
    for width, max_len in ((1600, 100000), (128, None), (40, None)):
        plans = [ops.paged_attention_plan(dtype, 8, 64, d, tokens, 8 * group, batch, width, max_len,
                                          bits=4) for batch in (tokens, tokens + 1, 64, 256, 100000)]
        assert all(p == plans[0] for p in plans), (width, plans)
    assert tokens > 5 or d * group > 512 or plans[0]["parts"] > 1


def test_workspace_of_a_padded_batch():
    """The parts of every window and of every smaller table or max_len fit what the whole takes."""
    info = (ctypes.c_int64 * 6)()
    L = _lib.lib()
    c = ctypes.byref(_lib.Mx4Cache(P, P, P, P, 4, 2, 64, 128))
    for dt in (CS_F32, CS_BF16):
        for tokens, batch in ((1, 7), (3, 256), (64, 4000)):
            for width in (1, 16, 100, 1024, 1500):
                need = L.cs_mx4_paged_attention_workspace_bytes(c, dt, tokens, 8, batch, width, 0)
                for less in (width, max(1, width - 1), max(1, width // 3)):
                    for max_len in (0, 1, less * 64 - 5, less * 64 + 1000):
                        for window in (0, 1, 1000, 4097, 50000):
                            assert L.cs_mx4_paged_attention_plan(c, dt, tokens, 8, batch, less,
                                                                 max_len, window, info) == CS_OK
                            assert info[5] <= need
