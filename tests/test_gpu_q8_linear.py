"""The linear layer on 8-bit codes against the 64-bit oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import q8_oracle as o8
from paper_2112_13896_amd import ops
from tests.q8_util import DTYPES, bound_linear, f64, rand

pytestmark = pytest.mark.gpu


def _codes(r, shape):
    return r.integers(-127, 128, size=shape).astype(np.int8)


def _strided(a: np.ndarray, ld: int, lead: int = 0) -> torch.Tensor:
    """The matrix on the GPU with row stride ld, `lead` bytes into its storage, among codes that
    must not matter."""
    buf = torch.full((a.shape[0] * ld + lead,), 113, dtype=torch.int8)
    view = buf[lead:].view(a.shape[0], ld)
    view[:, :a.shape[1]] = torch.from_numpy(a)
    return buf.cuda()[lead:].view(a.shape[0], ld)[:, :a.shape[1]]


def _check(y, qx, sx, qw, sw, bias, dt, what=""):
    ref, mag = o8.linear(qx, sx, qw, sw, bias)
    err, tol = np.abs(f64(y) - ref), bound_linear(ref, mag, dt)
    assert (err <= tol).all(), f"{what}: worst {np.max(err / tol)} of the bound"


SHAPES = [(1, 1, 1), (1, 16, 16), (1, 512, 512), (2, 100, 33), (3, 1000, 7), (5, 64, 300),
          (8, 4096, 48), (15, 333, 129), (16, 2048, 100), (17, 128, 257), (31, 65, 64),
          (33, 2048, 1000), (48, 640, 96), (64, 96, 65), (65, 129, 127), (100, 1500, 1001),
          (127, 63, 128), (128, 128, 128), (129, 192, 255), (255, 520, 256), (256, 256, 256),
          (257, 1024, 513), (300, 2049, 320), (512, 384, 1024), (700, 777, 260)]


@pytest.mark.parametrize("m,k,n", SHAPES)
def test_codes(m, k, n):
    """Row strides padded to 16 bytes (the fast way) and as odd as k."""
    r = np.random.default_rng(m * 7 + k * 3 + n)
    qx, qw = _codes(r, (m, k)), _codes(r, (n, k))
    sx = np.exp(r.standard_normal(m)).astype(np.float32)
    sw = np.exp(r.standard_normal(n)).astype(np.float32)
    bias = (100 * r.standard_normal(n)).astype(np.float32)
    pad = (k + 15) // 16 * 16
    dsx, dsw, db = (torch.from_numpy(a).cuda() for a in (sx, sw, bias))
    for ldx, ldw, lead in ((pad, pad, 0), (pad + 32, pad, 0), (k, k, 0), (k + 1, pad, 3)):
        for b, dbias in ((None, None), (bias, db)):
            y = ops.linear_q8(_strided(qx, ldx, lead), _strided(qw, ldw), dsw, sx=dsx, bias=dbias)
            _check(y, qx, sx, qw, sw, b, torch.float32, f"strides {ldx} {ldw}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,n", [(1, 512, 512), (3, 70, 40), (33, 2048, 1000), (140, 300, 333),
                                   (260, 1024, 512)])
def test_floats_in_and_out(dtype, m, k, n):
    """Tokens quantised in the call: the same codes as quantise_rows, each output type."""
    dt = DTYPES[dtype]
    r = np.random.default_rng(m + k + n)
    x = rand(r, (m, k), dt)
    w = rand(r, (n, k), torch.float32, 0.05)
    bias = r.standard_normal(n).astype(np.float32)
    qw, sw = ops.quantise_rows(w.cuda())
    qx, sx = o8.quantise(f64(x))
    ws = ops.linear_q8_workspace(dt, m, k, n)
    for out in (None, *DTYPES.values()):
        y = ops.linear_q8(x.cuda(), qw, sw, bias=torch.from_numpy(bias).cuda(), out_dtype=out,
                          ws=ws)
        assert y.dtype == (out or dt)
        _check(y, qx, sx, qw.cpu().numpy(), sw.cpu().numpy(), bias, y.dtype)
    wide = torch.full((m, n + 9), 5.0, dtype=dt, device="cuda")
    y2 = ops.linear_q8(x.cuda(), qw, sw, bias=torch.from_numpy(bias).cuda(), out=wide[:, 4:n + 4])
    assert torch.equal(y2, ops.linear_q8(x.cuda(), qw, sw, bias=torch.from_numpy(bias).cuda()))
    assert bool((wide[:, :4] == 5).all()) and bool((wide[:, n + 4:] == 5).all())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_largest_sums(m):
    """k at its limit with the largest codes: the sum nears 2^31."""
    k, n = 131072, 5
    qx = np.full((m, k), 127, dtype=np.int8)
    qw = np.full((n, k), -127, dtype=np.int8)
    qw[1] = 127
    qw[2, ::2] = 127
    sx, sw = np.ones(m, np.float32), np.full(n, 2.0 ** -20, np.float32)
    y = ops.linear_q8(torch.from_numpy(qx).cuda(), torch.from_numpy(qw).cuda(),
                      torch.from_numpy(sw).cuda(), sx=torch.from_numpy(sx).cuda())
    _check(y, qx, sx, qw, sw, None, torch.float32)


def test_a_token_that_is_not_finite():
    """Its outputs are NaN, no other token's are."""
    r = np.random.default_rng(3)
    w, sw = ops.quantise_rows(rand(r, (70, 96), torch.float32).cuda())
    for m in (5, 90):
        x = rand(r, (m, 96), torch.bfloat16)
        x[3, 50] = float("inf")
        x[1, 0] = float("nan")
        nan = torch.isnan(ops.linear_q8(x.cuda(), w, sw)).cpu()
        assert nan[[1, 3]].all() and nan.sum() == 2 * 70


def test_no_rows_and_zero_rows():
    r = np.random.default_rng(4)
    w, sw = ops.quantise_rows(rand(r, (10, 32), torch.float32).cuda())
    bias = torch.arange(10, dtype=torch.float32).cuda()
    assert ops.linear_q8(torch.empty((0, 32), device="cuda"), w, sw).shape == (0, 10)
    y = ops.linear_q8(torch.zeros((3, 32), device="cuda"), w, sw, bias=bias)
    assert torch.equal(y, bias.expand(3, 10))


def test_other_stream_and_graph():
    """Enqueued on torch's current stream; captured and replayed with other inputs."""
    r = np.random.default_rng(5)
    for m, k, n in ((2, 512, 96), (80, 300, 200), (512, 512, 512)):
        w, sw = ops.quantise_rows(rand(r, (n, k), torch.float32).cuda())
        xs = [rand(r, (m, k), torch.bfloat16).cuda() for _ in range(4)]
        want = [ops.linear_q8(x, w, sw) for x in xs]
        static, out = xs[0].clone(), torch.empty_like(want[0])
        ws = ops.linear_q8_workspace(static.dtype, m, k, n)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = ops.linear_q8(xs[1], w, sw)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, want[1])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.linear_q8(static, w, sw, ws=ws, out=out)
        for x, ref in zip(xs, want):
            static.copy_(x)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
            assert torch.equal(ops.linear_q8(x, w, sw), ref)


@pytest.mark.parametrize("m,k,n", [(1, 8192, 40), (1, 16384, 17), (2, 8192, 33), (3, 2731, 50),
                                   (5, 3276, 16), (16, 1024, 64), (16, 1025, 64), (20, 8192, 2048),
                                   (20, 900, 2064), (64, 8192, 128), (130, 8200, 70)])
def test_few_and_many_tokens_at_the_rules_edges(m, k, n):
    """Sizes on both sides of what is quantised in the product's launch, and of the tiles."""
    r = np.random.default_rng(m + k + n)
    x = rand(r, (m, k), torch.bfloat16)
    w = rand(r, (n, k), torch.float32, 0.05)
    qw, sw = ops.quantise_rows(w.cuda())
    qx, sx = o8.quantise(f64(x))
    y = ops.linear_q8(x.cuda(), qw, sw)
    _check(y, qx, sx, qw.cpu().numpy(), sw.cpu().numpy(), None, torch.bfloat16)
    shifted = torch.zeros((m, k + 3), dtype=torch.bfloat16).cuda()[:, 3:]
    shifted.copy_(x)
    assert torch.equal(ops.linear_q8(shifted, qw, sw), y)


def test_last_rows_end_with_their_storage():
    """k that is no multiple of 16 in storage that ends with the last code."""
    r = np.random.default_rng(8)
    for m, k, n in ((3, 100, 20), (70, 1500, 65), (300, 129, 300)):
        qx, qw = _codes(r, (m, k)), _codes(r, (n, k))
        ld = (k + 15) // 16 * 16

        def tight(a):
            buf = torch.full(((a.shape[0] - 1) * ld + k,), 99, dtype=torch.int8)
            view = buf.as_strided(a.shape, (ld, 1))
            view.copy_(torch.from_numpy(a))
            return buf.cuda().as_strided(a.shape, (ld, 1))
        sx, sw = np.ones(m, np.float32), np.ones(n, np.float32)
        y = ops.linear_q8(tight(qx), tight(qw), torch.from_numpy(sw).cuda(),
                          sx=torch.from_numpy(sx).cuda())
        _check(y, qx, sx, qw, sw, None, torch.float32)
