"""Scales of a cache start on 4 bytes, wherever else: every operator gives what it gives where they
start on 16."""
from __future__ import annotations

import pytest
import torch

from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, Sequences

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("off", [1, 2, 3])
def test_scales_off_16_bytes(dtype, off):
    for new in (1, 3, 70):
        s = Sequences(off, [(new, 300), (new, 75), (new, 2500)], 2, 2, 48, 16, DTYPES[dtype])
        q, cache, table, lens, starts = s.args()

        def moved(t):
            m = torch.empty(t.numel() + off, device="cuda")[off:].view(t.shape)
            assert m.data_ptr() % 16 == 4 * off
            return m.copy_(t)
        other = ops.PagedCache(cache.k.clone(), cache.v.clone(), moved(cache.k_scale),
                               moved(cache.v_scale))
        assert torch.equal(ops.paged_attention(q, other, table, lens, starts),
                           ops.paged_attention(q, cache, table, lens, starts))
        x = torch.randn((5, 2, 48), device="cuda").to(DTYPES[dtype])
        slots = torch.arange(5, device="cuda")
        for c in (cache, other):
            ops.cache_write(c, x, x, slots)
        for a, b in zip(ops.cache_read(cache, slots, q.dtype), ops.cache_read(other, slots, q.dtype)):
            assert torch.equal(a, b)
        live = ~torch.isnan(cache.k_scale)
        assert torch.equal(cache.k_scale[live], other.k_scale[live])
