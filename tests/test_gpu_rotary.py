"""Rotary positions against the 64-bit oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as o4
from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, ROUND, f64, rand

pytestmark = pytest.mark.gpu


def _bound(x, ref, amplitude, dtype):
    """Two products and their sum in 32 bits of factors rounded to 32 bits: sine and cosine are
    within 2^-22 (argument, series and amplitude: a rounding each, one step of 2^-23 of slack), the
    products and the sum add three roundings of 2^-24; then the output's own."""
    rel, tiny = ROUND[dtype]
    size = np.abs(x).max(axis=-1, keepdims=True) * abs(amplitude)
    return 2 * (2.0 ** -22 + 3 * 2.0 ** -24) * size + rel * np.abs(ref) * (1 + 2.0 ** -20) + tiny


def _check(got, x, positions, f, amplitude, interleaved, dtype, inverse=False):
    ref = o4.rotary(f64(x), positions.cpu().numpy(), f, amplitude, interleaved, inverse)
    err = np.abs(f64(got) - ref)
    # pairs are turned among themselves; a bound of the whole head's largest covers them
    bad = ~(err <= _bound(f64(x), ref, amplitude, dtype))
    assert not bad.any(), (np.argwhere(bad)[0], err.max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", [(1, 1, 1, 2, 2), (1, 32, 8, 128, 128),
                                                (5, 3, 1, 80, 40), (77, 4, 2, 64, 64),
                                                (9, 7, 7, 48, 26), (3, 2, 1, 256, 254),
                                                (2100, 3, 1, 32, 16), (2, 5, 3, 33, 10)])
def test_sizes(dtype, interleaved, tokens, hq, hk, d, rot):
    r = np.random.default_rng(tokens + d)
    dt = DTYPES[dtype]
    q, k = rand(r, (tokens, hq, d), dt), rand(r, (tokens, hk, d), dt)
    pos = torch.from_numpy(r.integers(0, 5000, tokens).astype(np.int32)).cuda()
    f, amplitude = ops.rotary_frequencies(rot)
    ro = ops.Rotary.make(rot, interleaved=interleaved)
    for got, x in zip(ops.rotary(ro, pos, q.cuda(), k.cuda()), (q, k)):
        _check(got, x, pos, f, amplitude, interleaved, dt)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Angles of positions up to 2^31 - 1 are formed without loss.  (The oracle's own angle, a
    64-bit product of up to 2^31 radians, is off by 2^-22 at the far end: positions up to 2^28.)"""
    r = np.random.default_rng(1)
    pos = torch.tensor([0, 1, 2 ** 20 + 1, 10 ** 6, 2 ** 24 + 1, 2 ** 28 - 1], dtype=torch.int32)
    x = rand(r, (6, 2, 64), torch.float32)
    for scaling, how in (("none", {}), ("bands", dict(factor=8.0, original=8192)),
                         ("ramp", dict(factor=16.0, original=4096)), ("linear", dict(factor=3.0)),
                         ("base", dict(factor=5.0))):
        f, amplitude = ops.rotary_frequencies(64, 10000.0, scaling, **how)
        ro = ops.Rotary.make(64, 10000.0, scaling=scaling, interleaved=interleaved, **how)
        _check(ops.rotary(ro, pos.cuda(), x.cuda()), x, pos, f, amplitude, interleaved,
               torch.float32)
    # a quarter of a turn a position: exact at any position
    ro = ops.Rotary.of([np.pi / 2], interleaved)
    y = torch.tensor([[[3.0, 5.0]]] * 4, device="cuda")
    pos = torch.tensor([2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 3, 2 ** 31 - 4], dtype=torch.int32)
    got = f64(ops.rotary(ro, pos.cuda(), y))[:, 0]
    want = np.array([[5, -3], [-3, -5], [-5, 3], [3, 5]])
    # the frequency itself is a 64-bit number: 2^31 positions of its error of 2^-54 of a turn
    assert np.abs(got - want).max() < 2.0 ** -20


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_strided_and_unaligned(dtype, interleaved):
    """Parts of one tensor turned where they are: the same bits, and nothing else is touched."""
    dt = DTYPES[dtype]
    r = np.random.default_rng(2)
    qkv = rand(r, (13, 9, 64), dt).cuda()
    pos = torch.arange(100, 113, dtype=torch.int32, device="cuda")
    ro = ops.Rotary.make(48, interleaved=interleaved)
    want = ops.rotary(ro, pos, qkv[:, :5].contiguous(), qkv[:, 5:7].contiguous())
    y = qkv.clone()
    q, k = y[:, :5], y[:, 5:7]
    got = ops.rotary(ro, pos, q, k, out=(q, k))
    assert got[0] is q
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(y[:, 7:], qkv[:, 7:])
    flat = torch.zeros(13 * 5 * 67 + 1, dtype=dt, device="cuda")
    odd = flat[1:].view(13, 5, 67)[:, :, 2:66]
    odd.copy_(qkv[:, :5])
    assert torch.equal(ops.rotary(ro, pos, odd), want[0])
    keep = flat.clone()
    ops.rotary(ro, pos, odd, out=odd)
    assert torch.equal(odd, want[0])
    flat[1:].view(13, 5, 67)[:, :, 2:66] = keep[1:].view(13, 5, 67)[:, :, 2:66]
    assert torch.equal(flat, keep)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """The inverse call is the gradient: against the transposed map in 64 bits, and against
    differences of the call itself (which is linear, so a difference over the whole step has no
    error but its roundings: 2^-22 of the sizes, summed over up to 8 channels)."""
    r = np.random.default_rng(3)
    x = torch.from_numpy(r.standard_normal((4, 2, 8))).float().cuda()
    g = torch.from_numpy(r.standard_normal((4, 2, 8))).float().cuda()
    pos = torch.tensor([0, 3, -1, 70000], dtype=torch.int32, device="cuda")
    how = dict(scaling="ramp", factor=4.0, original=64)
    ro = ops.Rotary.make(6, interleaved=interleaved, **how)
    f, amplitude = ops.rotary_frequencies(6, **how)
    back = ops.rotary(ro, pos, g, inverse=True)
    _check(back, g, pos, f, amplitude, interleaved, torch.float32, inverse=True)
    num = np.zeros(x.shape)
    for c in range(8):
        e = torch.zeros_like(x)
        e[..., c] = 1.0
        diff = f64(ops.rotary(ro, pos, x + e)) - f64(ops.rotary(ro, pos, x - e))
        num[..., c] = (f64(g) * diff).sum(-1) / 2
    assert np.abs(num - f64(back)).max() < 8 * 2.0 ** -22 * 8


def test_positions_below_zero_are_copied():
    x = torch.randn((3, 2, 32), device="cuda").half()
    pos = torch.tensor([-1, 5, -2 ** 31], dtype=torch.int32, device="cuda")
    y = ops.rotary(ops.Rotary.make(32), pos, x)
    assert torch.equal(y[0], x[0]) and torch.equal(y[2], x[2]) and not torch.equal(y[1], x[1])


def test_no_tokens_and_streams():
    ro = ops.Rotary.make(32)
    none = torch.empty((0, 2, 32), device="cuda")
    no_positions = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.rotary(ro, no_positions, none).shape == none.shape
    x = torch.randn((40, 2, 32), device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    want = ops.rotary(ro, pos, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.rotary(ro, pos, x)
    side.synchronize()
    assert torch.equal(got, want)
