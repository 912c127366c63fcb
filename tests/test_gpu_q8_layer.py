"""The attention layer that runs the 8-bit operators together: its steps are the operators', a
prompt in chunks gives what it gives whole, and all of it stays near the layer in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2112_13896_amd import ops
from paper_2112_13896_amd.attention import AttentionLayer, PagePool, Sequence, Step
from tests.q8_util import DTYPES, f64

pytestmark = pytest.mark.gpu

WIDTH, HEADS, Q_HEADS, D, PAGE = 200, 2, 6, 48, 16


def _weights(seed, dtype=torch.float32):
    r = np.random.default_rng(seed)
    return [torch.from_numpy(r.standard_normal(s) / math.sqrt(s[1])).to(dtype)
            for s in ((Q_HEADS * D, WIDTH), (HEADS * D, WIDTH), (HEADS * D, WIDTH),
                      (WIDTH, Q_HEADS * D))]


def _layer64(ws, x):
    wq, wk, wv, wo = (f64(w) for w in ws)
    x = f64(x)
    n, g = len(x), Q_HEADS // HEADS
    q, k, v = ((x @ w.T).reshape(n, -1, D) for w in (wq, wk, wv))
    out = np.zeros((n, Q_HEADS, D))
    for h in range(Q_HEADS):
        s = q[:, h] @ k[:, h // g].T / math.sqrt(D)
        s[np.triu_indices(n, 1)] = -np.inf
        e = np.exp(s - s.max(1, keepdims=True))
        out[:, h] = e / e.sum(1, keepdims=True) @ v[:, h // g]
    return out.reshape(n, -1) @ wo.T


@pytest.mark.parametrize("dtype", DTYPES)
def test_steps_are_the_operators(dtype):
    dt = DTYPES[dtype]
    layer = AttentionLayer(*_weights(1), HEADS, D, dtype=dt)
    pool, cache = PagePool(12, PAGE), layer.make_cache(12, PAGE)
    seqs = [Sequence(), Sequence(), Sequence()]
    new = [33, 1, 20]
    for s, n in zip(seqs, new):
        pool.extend(s, n)
    step = Step.of(seqs, new, PAGE)
    x = torch.from_numpy(np.random.default_rng(2).standard_normal((54, WIDTH))).to(dt).cuda()
    y = layer.forward(x, cache, step)
    qkv = ops.linear_q8(x, layer.wqkv, layer.sqkv).view(54, -1, D)
    other = layer.make_cache(12, PAGE)
    ops.cache_write(other, qkv[:, Q_HEADS:Q_HEADS + HEADS].contiguous(),
                    qkv[:, Q_HEADS + HEADS:].contiguous(), step.slots)
    for a, b in zip(ops.cache_read(cache, step.slots, dt), ops.cache_read(other, step.slots, dt)):
        assert torch.equal(a, b)
    o = ops.paged_attention(qkv[:, :Q_HEADS].contiguous(), other, step.table, step.lens,
                            step.starts)
    assert torch.equal(y, ops.linear_q8(o.view(54, -1), layer.wo, layer.so))
    buffers = layer.make_buffers(54, cache, step)
    assert torch.equal(layer.forward(x, cache, step, buffers), y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_prompt_whole_in_chunks_and_by_tokens(dtype):
    """Against the layer in 64 bits without any quantisation: a code is at most half a step, 1/254
    of its row's largest, off; with rows whose largest is some three times their size that is 0.7 %
    of the size, uniformly spread, so 0.4 % in the mean, for tokens and weights in each of the two
    products and for keys and values: six independent errors, 1 % together; keys' errors act
    through the softmax, doubled for that.  5 % of the norm leaves room, and a mistake shows as
    much more."""
    dt = DTYPES[dtype]
    ws = _weights(3)
    x = torch.from_numpy(np.random.default_rng(4).standard_normal((90, WIDTH))).to(dt)
    want = _layer64(ws, x)
    for chunks in ([90], [40, 49, 1], [1] * 90):
        layer = AttentionLayer(*ws, HEADS, D, dtype=dt)
        pool, cache = PagePool(6, PAGE), layer.make_cache(6, PAGE)
        seq, got, at = Sequence(), [], 0
        for n in chunks:
            pool.extend(seq, n)
            got.append(layer.forward(x[at:at + n].cuda(), cache, Step.of([seq], [n], PAGE)))
            at += n
        got = f64(torch.cat(got))
        assert np.linalg.norm(got - want) < 0.05 * np.linalg.norm(want), chunks
        pool.release(seq)
        assert len(pool) == 6


def test_refusals():
    ws = _weights(5)
    with pytest.raises(ValueError):
        AttentionLayer(ws[0], ws[1], ws[2][:-1], ws[3], HEADS, D)
    with pytest.raises(ValueError):
        AttentionLayer(ws[0], ws[1], ws[2], ws[3].t(), HEADS, D)
    layer = AttentionLayer(*ws, HEADS, D)
    with pytest.raises(TypeError):
        layer.forward(torch.zeros((1, WIDTH), device="cuda"), layer.make_cache(1, PAGE), None)
