"""An attention layer served in 8 bits, its cache in 8 or 4, and the plan of a step over many
sequences.

The layer runs the operators as they are meant to be used together:

  tokens -> linear_q8 (queries, keys and values in one product)
         -> rotary (queries and keys to their positions, where the layer has them)
         -> cache_write (the new tokens' keys and values, quantised per token and head)
         -> paged_attention (each sequence's new tokens over all its positions)
         -> linear_q8 (output projection)

Weights are quantised once (quantise_rows, a scale per output channel).  A Step
says which tokens of the batch belong to which sequence and where their keys
live; a prompt, a part of one, drafted tokens and a decoding step differ in
nothing but the number of new tokens.  It is made on the host (Step.of, with a
PagePool's pages) or on the GPU (Step.plan, with an ops.DevicePool's), where a
recorded graph can make the next one.  forward() only enqueues kernels on
torch's current stream; buffers that its caller wants to keep (for a recorded
graph, say) come from make_buffers().
"""
from __future__ import annotations

from dataclasses import dataclass, field

import numpy as np
import torch

from . import ops


@dataclass
class Sequence:
    """Pages and length of one sequence."""
    pages: list = field(default_factory=list)
    length: int = 0


class PagePool:
    """The free pages of a cache (host bookkeeping)."""

    def __init__(self, pages: int, page: int):
        self.page = page
        self._free = list(range(pages - 1, -1, -1))

    def __len__(self) -> int:
        return len(self._free)

    def extend(self, seq: Sequence, new: int) -> None:
        """Room for `new` more tokens of the sequence; raises (and takes nothing) when the pool
        has too few pages."""
        if new < 0:
            raise ValueError("new must not be negative")
        need = -(-(seq.length + new) // self.page) - len(seq.pages)
        if need > len(self._free):
            raise RuntimeError(f"{need} pages needed, {len(self._free)} free")
        for _ in range(need):
            seq.pages.append(self._free.pop())
        seq.length += new

    def release(self, seq: Sequence) -> None:
        """Take back every page of a sequence that has ended."""
        self._free.extend(reversed(seq.pages))
        seq.pages, seq.length = [], 0


@dataclass
class Step:
    """What paged_attention, cache_write and rotary need to know of a batch of new tokens."""
    table: torch.Tensor      # int32 [batch][pages]
    lens: torch.Tensor       # int32 [batch]
    starts: torch.Tensor     # int32 [batch + 1]
    slots: torch.Tensor      # int64 [tokens]
    max_len: int
    positions: torch.Tensor | None = None    # int32 [tokens]
    status: torch.Tensor | None = None       # int32 [2], of a step planned on the GPU

    @classmethod
    def of(cls, seqs, new, page: int, device="cuda", width: int = 0) -> "Step":
        """The step in which sequence i (its new tokens already in its length and pages) brings
        new[i] tokens; `width` pads the page table to a fixed number of columns."""
        if not seqs or len(seqs) != len(new):
            raise ValueError("one number of new tokens for each of at least one sequence")
        for s, n in zip(seqs, new):
            if not 0 <= n <= s.length or len(s.pages) * page < s.length:
                raise ValueError("a sequence lacks the tokens or pages that the step needs")
        batch, width = len(seqs), max(width, 1, max(len(s.pages) for s in seqs))
        tokens, fresh = int(sum(new)), np.array(new, dtype=np.int32)
        # parts of one buffer, so that a step is one copy to the device, positions among it
        sizes = (2 * tokens, batch * width, batch, batch + 1, tokens)
        host = np.empty(sum(sizes), dtype=np.int32)
        slots, table, lens, starts, positions = np.split(host, np.cumsum(sizes)[:-1])
        slots, table = slots.view(np.int64), table.reshape(batch, width)
        table.fill(-1)
        for i, s in enumerate(seqs):
            table[i, :len(s.pages)] = s.pages
        lens[:] = [s.length for s in seqs]
        starts[0] = 0
        np.cumsum(fresh, out=starts[1:])
        # token t of sequence i is at position t - starts[i] + lens[i] - new[i]
        positions[:] = np.arange(tokens) + np.repeat(lens - starts[1:], fresh)
        slots[:] = table[np.repeat(np.arange(batch), fresh), positions // page]
        slots *= page
        slots += positions % page
        slots, table, lens, starts, positions = torch.from_numpy(host).to(device).split(sizes)
        return cls(table.view(batch, width), lens, starts, slots.view(torch.int64),
                   max(s.length for s in seqs), positions)

    @classmethod
    def plan(cls, pool: ops.DevicePool, seqs: torch.Tensor, new: torch.Tensor, tokens: int,
             max_len: int, width: int | None = None, ws: torch.Tensor | None = None,
             into: "Step | None" = None) -> "Step":
        """The step in which new[i] tokens come to sequence seqs[i] of the pool, planned by a kernel
        (ops.plan_step): of up to `tokens` tokens, padded to that many, and sequences of up to
        max_len positions as far as the caller knows.  `into`: an earlier planned step of these sizes,
        overwritten and returned.  The step's status is 0, 0 unless the pool could not give it."""
        out = None
        if into is not None:
            if into.positions is None or into.status is None:
                raise ValueError("into must be a step planned on the GPU")
            out = (into.table, into.lens, into.starts, into.slots, into.positions, into.status)
        table, lens, starts, slots, positions, status = ops.plan_step(pool, seqs, new, tokens,
                                                                      width, ws, out)
        if into is not None:
            into.max_len = max_len
            return into
        return cls(table, lens, starts, slots, max_len, positions, status)


class AttentionLayer:
    """wq [q_heads * d][width], wk and wv [heads * d][width], wo [width][q_heads * d]: float
    weights, quantised here; biases (float32) or None.  `dtype`: the type of the tokens and of
    what is between the products.  `rotary`: what turns queries and keys to their positions."""

    def __init__(self, wq, wk, wv, wo, heads: int, d: int, *, bias=None, out_bias=None,
                 dtype: torch.dtype = torch.bfloat16, window: int = 0, device="cuda",
                 rotary: ops.Rotary | None = None):
        if wq.shape[0] % d or wk.shape[0] != heads * d or wv.shape != wk.shape or \
                wo.shape != (wq.shape[1], wq.shape[0]):
            raise ValueError("weights do not fit the heads")
        self.heads, self.d, self.q_heads = heads, d, wq.shape[0] // d
        if self.q_heads % heads:
            raise ValueError("query heads must be a multiple of the cache's heads")
        if rotary is not None and rotary.rot > d:
            raise ValueError("rotary positions turn more channels than a head has")
        self.width, self.dtype, self.window, self.rotary = wq.shape[1], dtype, window, rotary
        self.device = torch.device(device)

        def weights(w):
            return ops.quantise_rows(w.to(self.device).contiguous())
        self.wqkv, self.sqkv = weights(torch.cat([wq, wk, wv]))
        self.wo, self.so = weights(wo)
        self.bias = None if bias is None else bias.to(self.device, torch.float32)
        self.out_bias = None if out_bias is None else out_bias.to(self.device, torch.float32)

    def make_cache(self, pages: int, page: int = 64, bits: int = 8) -> ops.PagedCache:
        if bits not in (8, 4):
            raise ValueError("a cache has 8 or 4 bits")
        kind = ops.PagedCache if bits == 8 else ops.PagedCache4
        return kind.empty(pages, self.heads, page, self.d, self.device)

    def make_buffers(self, tokens: int, cache: ops.PagedCache, step: Step) -> dict:
        """Intermediates and workspaces of forward() for this many tokens and such a step."""
        def empty(*shape):
            return torch.empty(shape, dtype=self.dtype, device=self.device)
        q = empty(tokens, self.q_heads, self.d)
        n_qkv, n_o = self.wqkv.shape[0], self.q_heads * self.d
        return dict(qkv=empty(tokens, n_qkv), o=q, y=empty(tokens, self.width),
                    ws_qkv=ops.linear_q8_workspace(self.dtype, tokens, self.width, n_qkv,
                                                   self.device),
                    ws_att=ops.paged_attention_workspace(q, cache, step.table, step.max_len),
                    ws_o=ops.linear_q8_workspace(self.dtype, tokens, n_o, self.width, self.device))

    def forward(self, x: torch.Tensor, cache: ops.PagedCache, step: Step,
                buffers: dict | None = None) -> torch.Tensor:
        """x [tokens][width] of the step's new tokens -> [tokens][width]; the cache gains their
        keys and values."""
        if x.dtype != self.dtype:
            raise TypeError(f"tokens must be {self.dtype}")
        if self.rotary is not None and step.positions is None:
            raise ValueError("the layer's rotary positions need the step's positions")
        b = buffers or {}
        qkv = ops.linear_q8(x, self.wqkv, self.sqkv, bias=self.bias, out=b.get("qkv"),
                            ws=b.get("ws_qkv"))
        heads = qkv.unflatten(1, (-1, self.d))
        q, k, v = heads.split([self.q_heads, self.heads, self.heads], dim=1)
        if self.rotary is not None:
            ops.rotary(self.rotary, step.positions, q, k, out=(q, k))
        ops.cache_write(cache, k, v, step.slots)
        o = ops.paged_attention(q, cache, step.table, step.lens, step.starts, window=self.window,
                                max_len=step.max_len, out=b.get("o"), ws=b.get("ws_att"))
        return ops.linear_q8(o.flatten(1), self.wo, self.so, bias=self.out_bias, out=b.get("y"),
                             ws=b.get("ws_o"))
