"""The 8-bit attention-layer operators without a GPU: refusals of the C ABI and of the Python
wrappers (every check runs before the first HIP call), workspace sizes, and the oracle's own
definition on hand-made rows."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

from oracle import q8_oracle as o8
from paper_2112_13896_amd import _lib, ops
from paper_2112_13896_amd._lib import (CS_BF16, CS_ERR_ARG, CS_ERR_DTYPE, CS_ERR_SHAPE,
                                       CS_ERR_WORKSPACE, CS_F16, CS_F32, CS_I8, CS_I32, CS_OK)

P = 0x100000            # an aligned address that must never be dereferenced


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def _cache(k=P, v=P, ks=P, vs=P, pages=4, heads=2, page=16, d=64):
    return ctypes.byref(_lib.Q8Cache(k, v, ks, vs, pages, heads, page, d))


def test_quantise_refusals(L):
    def call(xt=CS_F32, x=P, ldx=64, rows=4, c=64, q=P, ldq=64, scale=P):
        return L.cs_quantise_rows(xt, x, ldx, rows, c, q, ldq, scale, None)
    for xt in (CS_I8, CS_I32, 9, -1):
        assert call(xt=xt) == CS_ERR_DTYPE
    for kw in (dict(x=0), dict(q=0), dict(scale=0), dict(rows=-1), dict(c=0), dict(x=P + 2),
               dict(scale=P + 1)):
        assert call(**kw) == CS_ERR_ARG, kw
    assert call(xt=CS_BF16, x=P + 1) == CS_ERR_ARG
    for kw in (dict(ldx=63), dict(ldq=63), dict(rows=1 << 31)):
        assert call(**kw) == CS_ERR_SHAPE, kw
    assert call(rows=0, x=0, q=0, scale=0) == CS_OK


def test_linear_refusals(L):
    def call(xt=CS_I8, x=P, ldx=64, sx=P, rows=4, k=64, w=P, ldw=64, sw=P, d_out=32, bias=0,
             yt=CS_F32, y=P, ldy=32, ws=P, n=1 << 30):
        return L.cs_linear_q8(xt, x, ldx, sx, rows, k, w, ldw, sw, d_out, bias, yt, y, ldy, ws, n,
                              None)
    for kw in (dict(xt=CS_I32), dict(xt=7), dict(yt=CS_I8), dict(yt=CS_I32), dict(yt=-2)):
        assert call(**kw) == CS_ERR_DTYPE, kw
    for kw in (dict(x=0), dict(w=0), dict(sw=0), dict(y=0), dict(sx=0), dict(rows=-1), dict(k=0),
               dict(d_out=0), dict(xt=CS_F32), dict(xt=CS_F16, sx=0, x=P + 1), dict(y=P + 2),
               dict(sw=P + 2), dict(bias=P + 3), dict(sx=P + 2)):
        assert call(**kw) == CS_ERR_ARG, kw
    for kw in (dict(ldx=63), dict(ldw=63), dict(ldy=31), dict(rows=1 << 31),
               dict(k=131073, ldx=131073, ldw=131073), dict(d_out=(1 << 22) + 1, ldy=1 << 23)):
        assert call(**kw) == CS_ERR_SHAPE, kw
    need = L.cs_linear_q8_workspace_bytes(CS_F32, 4, 64, 32)
    assert need >= 4 * 64 + 4 * 4
    for kw in (dict(ws=0), dict(n=need - 1), dict(ws=P + 8)):
        assert call(xt=CS_F32, sx=0, **kw) == CS_ERR_WORKSPACE, kw
    assert call(rows=0, x=0, w=0) == CS_OK
    for args in ((CS_F32, 0, 64, 32), (CS_F32, 4, 0, 32), (CS_F32, 4, 131073, 32), (CS_I32, 4, 4, 4),
                 (CS_F32, 4, 64, (1 << 22) + 1)):
        assert L.cs_linear_q8_workspace_bytes(*args) == 0


def test_cache_refusals(L):
    def write(c=None, xt=CS_F32, k=P, ldk=128, hsk=64, v=P, ldv=128, hsv=64, slots=P, tokens=3):
        return L.cs_cache_write(c or _cache(), xt, k, ldk, hsk, v, ldv, hsv, slots, tokens, None)

    def read(c=None, slots=P, tokens=3, yt=CS_F32, k=P, v=P):
        return L.cs_cache_read(c or _cache(), slots, tokens, yt, k, v, None)
    for f in (write, read):
        for kw in (dict(k=0), dict(v=0), dict(ks=0), dict(vs=0), dict(pages=0), dict(heads=0),
                   dict(page=0), dict(d=0), dict(k=P + 8), dict(v=P + 4), dict(ks=P + 2)):
            assert f(_cache(**kw)) == CS_ERR_ARG, kw
        for kw in (dict(d=24), dict(d=8), dict(d=272), dict(page=8), dict(page=48),
                   dict(page=2048), dict(pages=1 << 27, page=16)):
            assert f(_cache(**kw)) == CS_ERR_SHAPE, kw
        assert f(tokens=1 << 31) == CS_ERR_SHAPE
        for kw in (dict(k=0), dict(v=0), dict(slots=0), dict(tokens=-1), dict(slots=P + 4)):
            assert f(**kw) == CS_ERR_ARG, kw
        assert f(tokens=0, k=0, v=0, slots=0) == CS_OK
    assert L.cs_cache_write(None, CS_F32, P, 128, 64, P, 128, 64, P, 1, None) == CS_ERR_ARG
    assert write(xt=CS_I8) == CS_ERR_DTYPE and read(yt=CS_I32) == CS_ERR_DTYPE
    for kw in (dict(ldk=-1), dict(ldv=-1), dict(hsk=63), dict(hsv=63)):
        assert write(**kw) == CS_ERR_SHAPE, kw
    assert write(xt=CS_BF16, k=P + 1) == CS_ERR_ARG and read(k=P + 8) == CS_ERR_ARG


def test_attention_refusals(L):
    def call(c=None, qt=CS_BF16, q=P, ldq=256, hsq=64, tokens=5, q_heads=4, batch=2, table=P,
             width=3, lens=P, starts=P, max_len=0, scale=0.1, window=0, out=P, ws=P, n=1 << 40):
        return L.cs_paged_attention(c or _cache(), qt, q, ldq, hsq, tokens, q_heads, batch, table,
                                    width, lens, starts, max_len, scale, window, out, ws, n, None)
    for qt in (CS_I8, CS_I32, 11):
        assert call(qt=qt) == CS_ERR_DTYPE
    for kw in (dict(q=0), dict(table=0), dict(lens=0), dict(starts=0), dict(out=0), dict(tokens=-1),
               dict(q_heads=0), dict(batch=0), dict(width=0), dict(max_len=-1), dict(window=-1),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(q=P + 1), dict(out=P + 2), dict(table=P + 1),
               dict(lens=P + 2), dict(starts=P + 3)):
        assert call(**kw) == CS_ERR_ARG, kw
    for kw in (dict(q_heads=3), dict(ldq=-1), dict(hsq=63), dict(tokens=1 << 30),
               dict(width=1 << 27)):
        assert call(**kw) == CS_ERR_SHAPE, kw
    assert call(_cache(page=20)) == CS_ERR_SHAPE and call(_cache(k=0)) == CS_ERR_ARG
    assert call(tokens=0, q=0) == CS_OK
    # one token of a long sequence is split, and the parts need room
    big = dict(tokens=1, batch=1, width=4096)
    need = L.cs_paged_attention_workspace_bytes(_cache(), CS_BF16, 1, 4, 1, 4096, 0)
    if need:
        assert call(**big, n=need - 1) == CS_ERR_WORKSPACE
        assert call(**big, ws=0) == CS_ERR_WORKSPACE
        assert call(**big, ws=P + 8) == CS_ERR_WORKSPACE
    for args in ((CS_I8, 1, 4, 1, 4, 0), (CS_BF16, 0, 4, 1, 4, 0), (CS_BF16, 1, 3, 1, 4, 0),
                 (CS_BF16, 1, 4, 0, 4, 0), (CS_BF16, 1, 4, 1, 0, 0)):
        assert L.cs_paged_attention_workspace_bytes(_cache(), *args) == 0


def test_wrapper_refusals():
    f = torch.zeros
    cpu = ops.PagedCache.empty(2, 2, 16, 32, device="cpu")
    with pytest.raises(ValueError):
        ops.quantise_rows(f(4, 8))                            # not on a GPU
    with pytest.raises(ValueError):
        ops.linear_q8(f(4, 8), f(4, 8, dtype=torch.int8), f(4))
    with pytest.raises(ValueError):
        ops.cache_write(cpu, f(1, 2, 32), f(1, 2, 32), f(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        ops.paged_attention(f(1, 2, 48), cpu, f(1, 1, dtype=torch.int32),
                            f(1, dtype=torch.int32), f(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        ops.paged_attention_workspace(f(1, 2, 32, dtype=torch.int8), cpu,
                                      f(1, 1, dtype=torch.int32))
    with pytest.raises(TypeError):
        ops.linear_q8_workspace(torch.int32, 1, 1, 1, device="cpu")
    with pytest.raises(ValueError):
        ops.PagedCache(cpu.k, cpu.v, cpu.k_scale, cpu.v_scale[:1])
    with pytest.raises(ValueError):
        ops.PagedCache(cpu.k, cpu.v.float(), cpu.k_scale, cpu.v_scale)
    with pytest.raises(ValueError):
        ops.PagedCache(cpu.k[..., ::2], cpu.v[..., ::2], cpu.k_scale, cpu.v_scale)


def test_oracle_codes():
    x = np.array([[127.0, 0.5, 1.5, -2.5, 63.49, -126.5], [0, 0, 0, 0, 0, 0],
                  [1, np.nan, 0, 0, 0, 0], [-np.inf, 1, 0, 0, 0, 0]])
    q, s = o8.quantise(x)
    assert q[0].tolist() == [127, 0, 2, -2, 63, -126]
    assert not q[1:].any()
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2:]).all()


def test_oracle_attention():
    """Two keys of equal logits average their values; a token before both sees nothing."""
    k = np.zeros((2, 1, 16))
    v = np.stack([np.full((1, 16), 2.0), np.full((1, 16), 4.0)])
    q = np.ones((3, 1, 16))
    o, spread, logit, peak = o8.attention(q, [k], [v], np.array([2]), np.array([0, 3]), 1.0)
    assert (o[0] == 0).all() and (o[1] == 2).all() and (o[2] == 3).all()
    assert (spread[2] == 3).all() and (logit == 0).all() and peak[2] == 2
    o, *_ = o8.attention(q, [k], [v], np.array([2]), np.array([0, 3]), 1.0, window=1)
    assert (o[2] == 4).all()
