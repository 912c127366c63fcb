"""An attention layer served in 8 bits, and the plan of a step over many sequences.

The layer runs the four 8-bit operators as they are meant to be used together:

  tokens -> linear_q8 (queries, keys and values in one product)
         -> cache_write (the new tokens' keys and values, a scale per token and head)
         -> paged_attention (each sequence's new tokens over all its positions)
         -> linear_q8 (output projection)

Weights are quantised once (quantise_rows, a scale per output channel).  A Step
says which tokens of the batch belong to which sequence and where their keys
live; a prompt, a part of one, drafted tokens and a decoding step differ in
nothing but the number of new tokens.  forward() only enqueues kernels on
torch's current stream; buffers that its caller wants to keep (for a recorded
graph, say) come from make_buffers().
"""
from __future__ import annotations

from dataclasses import dataclass, field

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
    """What paged_attention and cache_write need to know of a batch of new tokens."""
    table: torch.Tensor      # int32 [batch][pages]
    lens: torch.Tensor       # int32 [batch]
    starts: torch.Tensor     # int32 [batch + 1]
    slots: torch.Tensor      # int64 [tokens]
    max_len: int

    @classmethod
    def of(cls, seqs, new, page: int, device="cuda", width: int = 0) -> "Step":
        """The step in which sequence i (its new tokens already in its length and pages) brings
        new[i] tokens; `width` pads the page table to a fixed number of columns."""
        if not seqs or len(seqs) != len(new):
            raise ValueError("one number of new tokens for each of at least one sequence")
        for s, n in zip(seqs, new):
            if not 0 <= n <= s.length or len(s.pages) * page < s.length:
                raise ValueError("a sequence lacks the tokens or pages that the step needs")
        width = max(width, 1, max(len(s.pages) for s in seqs))
        table = torch.full((len(seqs), width), -1, dtype=torch.int32)
        starts = torch.zeros(len(seqs) + 1, dtype=torch.int32)
        slots = []
        for i, (s, n) in enumerate(zip(seqs, new)):
            table[i, :len(s.pages)] = torch.tensor(s.pages, dtype=torch.int32)
            starts[i + 1] = starts[i] + n
            slots += [s.pages[j // page] * page + j % page for j in range(s.length - n, s.length)]
        lens = torch.tensor([s.length for s in seqs], dtype=torch.int32)
        return cls(table.to(device), lens.to(device), starts.to(device),
                   torch.tensor(slots, dtype=torch.int64).to(device),
                   max(s.length for s in seqs))


class AttentionLayer:
    """wq [q_heads * d][width], wk and wv [heads * d][width], wo [width][q_heads * d]: float
    weights, quantised here; biases (float32) or None.  `dtype`: the type of the tokens and of
    what is between the products."""

    def __init__(self, wq, wk, wv, wo, heads: int, d: int, *, bias=None, out_bias=None,
                 dtype: torch.dtype = torch.bfloat16, window: int = 0, device="cuda"):
        if wq.shape[0] % d or wk.shape[0] != heads * d or wv.shape != wk.shape or \
                wo.shape != (wq.shape[1], wq.shape[0]):
            raise ValueError("weights do not fit the heads")
        self.heads, self.d, self.q_heads = heads, d, wq.shape[0] // d
        if self.q_heads % heads:
            raise ValueError("query heads must be a multiple of the cache's heads")
        self.width, self.dtype, self.window = wq.shape[1], dtype, window
        self.device = torch.device(device)

        def weights(w):
            return ops.quantise_rows(w.to(self.device).contiguous())
        self.wqkv, self.sqkv = weights(torch.cat([wq, wk, wv]))
        self.wo, self.so = weights(wo)
        self.bias = None if bias is None else bias.to(self.device, torch.float32)
        self.out_bias = None if out_bias is None else out_bias.to(self.device, torch.float32)

    def make_cache(self, pages: int, page: int = 64) -> ops.PagedCache:
        return ops.PagedCache.empty(pages, self.heads, page, self.d, self.device)

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
        b = buffers or {}
        qkv = ops.linear_q8(x, self.wqkv, self.sqkv, bias=self.bias, out=b.get("qkv"),
                            ws=b.get("ws_qkv"))
        heads = qkv.unflatten(1, (-1, self.d))
        q, k, v = heads.split([self.q_heads, self.heads, self.heads], dim=1)
        ops.cache_write(cache, k, v, step.slots)
        o = ops.paged_attention(q, cache, step.table, step.lens, step.starts, window=self.window,
                                max_len=step.max_len, out=b.get("o"), ws=b.get("ws_att"))
        return ops.linear_q8(o.flatten(1), self.wo, self.so, bias=self.out_bias, out=b.get("y"),
                             ws=b.get("ws_o"))
