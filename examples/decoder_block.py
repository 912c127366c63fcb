"""A decoder block: attention in 8 bits over a paged 8-bit cache, then the
sparse-sparse feed-forward layers of this package, in fp32.

    python examples/decoder_block.py [--batch 16] [--prompt 300] [--tokens 32]

Prompts of different lengths are taken in chunks, then the sequences decode one
token at a time; the decoding step is recorded into a HIP graph once and
replayed.  Weights are random; the printed error compares the attention layer
with the same layer in 32-bit floats, nothing quantised.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.abspath(os.path.join(os.path.dirname(__file__), "..")))

from paper_2112_13896_amd.attention import AttentionLayer, PagePool, Sequence, Step  # noqa: E402
from paper_2112_13896_amd.network import Network  # noqa: E402
from workloads import LayerSpec, complementary_weights  # noqa: E402

WIDTH, HEADS, Q_HEADS, D, HIDDEN, PAGE = 512, 2, 8, 64, 2048, 64


def feed_forward(batch: int) -> Network:
    """width -> hidden with k-WTA -> width, kernels overlaid 8 to one, fp32."""
    r = np.random.default_rng(1)
    layers = [LayerSpec("up", "linear", WIDTH, HIDDEN, 8, k=HIDDEN // 10, weight_dist="normal"),
              LayerSpec("down", "linear", HIDDEN, WIDTH, 8, weight_dist="normal")]
    weights = [complementary_weights(r, r, s.c_out, s.r, s.n, "normal") for s in layers]
    return Network(layers, weights, [None, None], (WIDTH,), batch, keep_sums=False)


class Block:
    def __init__(self, seed: int = 0):
        g = torch.Generator().manual_seed(seed)

        def w(n, k):
            return torch.randn((n, k), generator=g) / math.sqrt(k)
        self.float_weights = [w(Q_HEADS * D, WIDTH), w(HEADS * D, WIDTH), w(HEADS * D, WIDTH),
                              w(WIDTH, Q_HEADS * D)]
        self.attention = AttentionLayer(*self.float_weights, HEADS, D, dtype=torch.float32)
        self.ffs = {}

    def forward(self, x, cache, step, buffers=None):
        y = x + self.attention.forward(x, cache, step, buffers)
        n = x.shape[0]
        if n not in self.ffs:
            self.ffs[n] = feed_forward(n)
        return y + self.ffs[n].forward(y)


def plain_attention(weights, x):
    """The layer on one whole sequence x [n][width] in 32-bit floats."""
    wq, wk, wv, wo = (w.to(x.device) for w in weights)
    n = x.shape[0]
    q = (x @ wq.t()).view(n, HEADS, Q_HEADS // HEADS, D)
    k, v = (x @ wk.t()).view(n, HEADS, D), (x @ wv.t()).view(n, HEADS, D)
    out = torch.empty((n, HEADS, Q_HEADS // HEADS, D), device=x.device)
    hidden = torch.ones((n, n), device=x.device).triu(1).bool()
    for h in range(HEADS):
        for j in range(Q_HEADS // HEADS):
            s = (q[:, h, j] @ k[:, h].t().contiguous()) / math.sqrt(D)
            out[:, h, j] = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1) @ v[:, h]
    return out.reshape(n, -1) @ wo.t()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=300, help="longest prompt")
    ap.add_argument("--tokens", type=int, default=32, help="decoding steps")
    a = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("this example needs a GPU")
    r = np.random.default_rng(2)
    lengths = [int(n) for n in r.integers(1, a.prompt + 1, size=a.batch)]
    width = -(-(a.prompt + a.tokens) // PAGE)
    block = Block()
    pool = PagePool(a.batch * width, PAGE)
    cache = block.attention.make_cache(a.batch * width, PAGE)
    seqs = [Sequence() for _ in lengths]
    prompts = [torch.from_numpy(r.standard_normal((n, WIDTH))).float().cuda() for n in lengths]

    # prompts in chunks of up to 128 tokens, all sequences in one call
    error = None
    last = [None] * a.batch
    for first in range(0, max(lengths), 128):
        new = [max(0, min(128, n - first)) for n in lengths]
        for s, n in zip(seqs, new):
            pool.extend(s, n)
        x = torch.cat([p[first:first + n] for p, n in zip(prompts, new)])
        step = Step.of(seqs, new, PAGE)
        if first == 0:
            got = block.attention.forward(x, cache, step)[:new[0]]
            want = plain_attention(block.float_weights, prompts[0][:new[0]])
            error = float((got - want).norm() / want.norm())
        y = block.forward(x, cache, step)
        for i, n in enumerate(new):
            if n:
                last[i] = y[int(step.starts[i]) + n - 1]
    x = torch.stack(last)

    # decoding: the step's tensors stay where they are, their contents change
    for s in seqs:
        pool.extend(s, 1)
    step = Step.of(seqs, [1] * a.batch, PAGE, width=width)
    step.max_len = a.prompt + a.tokens
    buffers = block.attention.make_buffers(a.batch, cache, step)
    static = x.clone()
    block.forward(static, cache, step, buffers)              # kernels loaded before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.forward(static, cache, step, buffers)
    began = time.perf_counter()
    for i in range(a.tokens):
        if i:
            for s in seqs:
                pool.extend(s, 1)
            now = Step.of(seqs, [1] * a.batch, PAGE, width=width)
            step.table.copy_(now.table)
            step.lens.copy_(now.lens)
            step.slots.copy_(now.slots)
        graph.replay()
        static.copy_(out / out.norm(dim=1, keepdim=True) * math.sqrt(WIDTH))
    torch.cuda.synchronize()
    s = (time.perf_counter() - began) / a.tokens
    print(f"attention layer against 32-bit floats: {error:.4f} of the norm")
    print(f"{a.batch} sequences of up to {a.prompt + a.tokens} positions: {1e6 * s:.0f} us a "
          f"decoding step, {a.batch / s:.0f} tokens/s")
    if not (error < 0.05 and bool(torch.isfinite(out).all())):
        raise SystemExit("the block's outputs are wrong")


if __name__ == "__main__":
    main()
