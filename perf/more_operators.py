"""The operators of an attention layer served over a 4-bit cache, as measurable cases.

"kind" names the operator:

  plan       a step over many sequences planned on the GPU: pages taken from a pool's free stack,
             then page table, lengths, first tokens, slots and positions of the new tokens; after
             it the tokens are taken back (drafts that were not accepted, a prompt that ended)
  rotary     rotary positions of a step's queries and keys, parts of one tensor as a projection
             leaves them
  cache      new tokens' keys and values quantised into a paged 4-bit cache (groups of 32 channels
             with a power of two each), then a stretch of the cache, the new tokens among it, read
             back as floats
  attention  a chunk of new tokens of each of several sequences against the paged 4-bit cache that
             holds them and their history; one new token a sequence is a decoding step

The plain forms are elementary torch operations in 32 bits, angles in 64.  Codes and scales are
part of an operator's definition: the scale of a group is the least power of two 2^E, E in
[-60, 60], with max|x| <= 7 * 2^E, and a code the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to
|x| / 2^E (ties to the even code) with the value's sign.  The pages that a step takes are part of
it too: the stack's top first, sequence after sequence.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # a decoding step of a small server: one token a sequence, latency
        dict(name="plan_64", kind="plan", batch=64, spare=32, new_lo=1, new_hi=1, past_hi=8191,
             page=64, width=160, ragged=1),
        # many sequences, chunks of prompts among them, small pages; odd numbers
        dict(name="plan_1001", kind="plan", batch=1001, spare=77, new_lo=0, new_hi=121,
             past_hi=6000, page=16, width=600, ragged=2),
        # one token: latency
        dict(name="rope_1", kind="rotary", tokens=1, q_heads=32, kv_heads=8, d=128, rot=128,
             interleaved=False, scaling="none", far=4096, dtype="bf16"),
        # part of an odd head in neighbouring pairs, odd numbers of heads and tokens
        dict(name="rope_777_d80", kind="rotary", tokens=777, q_heads=15, kv_heads=5, d=80, rot=40,
             interleaved=True, scaling="ramp", far=20000, dtype="f32"),
        # prompts far into a long context
        dict(name="rope_16384", kind="rotary", tokens=16384, q_heads=32, kv_heads=8, d=128,
             rot=128, interleaved=False, scaling="bands", far=1000000, dtype="bf16"),
        # a decoding step's tokens, each to its own sequence's page
        dict(name="cache4_48", kind="cache", tokens=48, read=48, heads=8, d=128, page=16,
             dtype="bf16"),
        # prompts written, twice as much read back (a prefix that two batches share)
        dict(name="cache4_16384", kind="cache", tokens=16384, read=32768, heads=8, d=128, page=64,
             dtype="f16"),
        # one sequence's next token, a short history: latency
        dict(name="attn4_1x1500", kind="attention", batch=1, new_lo=1, new_hi=1, past_lo=1500,
             past_hi=1500, kv_heads=8, group=4, d=128, page=16, window=0, dtype="bf16", ragged=1),
        # a server's decoding step: sequences of all lengths
        dict(name="attn4_96x12000", kind="attention", batch=96, new_lo=1, new_hi=1, past_lo=0,
             past_hi=12000, kv_heads=8, group=4, d=128, page=64, window=0, dtype="bf16", ragged=2),
        # few long sequences, five drafted tokens each to be checked
        dict(name="attn4_3x100000", kind="attention", batch=3, new_lo=5, new_hi=5, past_lo=70000,
             past_hi=100000, kv_heads=8, group=4, d=128, page=128, window=0, dtype="f16",
             ragged=3),
        # chunks of prompts among decoding sequences, odd heads, a sliding window, fp32
        dict(name="attn4_mixed_d80", kind="attention", batch=11, new_lo=1, new_hi=600, past_lo=0,
             past_hi=4000, kv_heads=5, group=3, d=80, page=32, window=777, dtype="f32", ragged=4),
        # whole prompts and continued ones
        dict(name="attn4_prompt_5x2000", kind="attention", batch=5, new_lo=2000, new_hi=2000,
             past_lo=0, past_hi=4096, kv_heads=8, group=4, d=128, page=64, window=0, dtype="bf16",
             ragged=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("plan", "rotary", "cache", "attention", "attention"))
    top = [work(c) for c in listed() if c["kind"] == kind]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while True:
        c = _draw_kind(rng, kind)
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _draw_kind(rng, kind):
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "plan":
        batch = _log_int(rng, 1, 1024)
        hi = rng.choice((1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 4096)))
        past = _log_int(rng, 16, 12000)
        return dict(kind=kind, batch=batch, spare=rng.randint(0, 100),
                    new_lo=rng.choice((0, 1, hi)), new_hi=hi, past_hi=past, page=page,
                    width=-(-(past + hi) // page) + rng.randint(0, 50),
                    ragged=rng.randint(0, 10 ** 6))
    if kind == "rotary":
        kv = rng.choice((1, 2, 3, 4, 5, 8, 16))
        d = 16 * rng.randint(1, 16)
        return dict(kind=kind, tokens=_log_int(rng, 1, 16384),
                    q_heads=kv * rng.choice((1, 3, 4, 8)), kv_heads=kv, d=d,
                    rot=rng.choice((d, d, 2 * rng.randint(1, d // 2))),
                    interleaved=rng.random() < 0.5,
                    scaling=rng.choice(("none", "linear", "base", "bands", "ramp")),
                    far=_log_int(rng, 16, 2000000), dtype=dtype)
    if kind == "cache":
        tokens = _log_int(rng, 1, 16384)
        more = rng.choice((0, _log_int(rng, 1, 16384)))
        return dict(kind=kind, tokens=tokens, read=tokens + more, heads=_log_int(rng, 1, 32),
                    d=16 * rng.randint(1, 16), page=page, dtype=dtype)
    mode = rng.choice(("one", "one", "draft", "chunk", "prompt"))
    batch = _log_int(rng, 1, 128 if mode == "one" else 16)
    lo = _log_int(rng, 1, 400)
    new = {"one": (1, 1), "draft": (2, rng.randint(2, 8)), "chunk": (lo, lo + rng.randint(0, 300)),
           "prompt": (1, _log_int(rng, 64, 2048))}[mode]
    hi = _log_int(rng, 16, 100000 if mode in ("one", "draft") else 8192)
    return dict(kind=kind, batch=batch, new_lo=new[0], new_hi=new[1],
                past_lo=rng.choice((0, hi // 2, hi)), past_hi=hi,
                kv_heads=rng.choice((1, 2, 3, 4, 5, 8, 16)), group=rng.choice((1, 2, 3, 4, 7, 8)),
                d=rng.choice((16, 32, 48, 64, 80, 96, 112, 128, 128, 128, 256)), page=page,
                window=rng.choice((0, 0, 0, _log_int(rng, 16, 4096))), dtype=dtype,
                ragged=rng.randint(0, 10 ** 6))


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """[(new tokens, tokens in the cache with them)] of the case's sequences."""
    r = random.Random(case["ragged"])
    out = []
    for _ in range(case["batch"]):
        n = r.randint(case["new_lo"], case["new_hi"])
        out.append((n, r.randint(case.get("past_lo", 0), case["past_hi"]) + n))
    return out


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tokens(gen, rows, c, dtype):
    """Activations as layers see them: tokens of different size, one channel in a hundred ten
    times as large as the others."""
    x = torch.randn((rows, c), generator=gen, device="cuda")
    x *= 1 + 9 * (torch.rand((c,), generator=gen, device="cuda") < 0.01)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    return x.to(dtype)


def _codes(gen, shape):
    """Bytes of two codes of normal values each, the largest of a group near the code of 6."""
    z = np.sqrt(2.0) * np.array([float(t) for t in torch.erfinv(
        (torch.arange(256, dtype=torch.float64) + 0.5) / 128 - 1)])
    edges = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
    code = np.searchsorted(edges, np.abs(z) * 2.2) + 8 * (z < 0)
    table = torch.from_numpy(code.astype(np.uint8)).cuda()
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 26):             # a piece at a time: indices are wide
        n = min(1 << 26, flat.numel() - i)
        pick = torch.randint(0, 256, (2, n), generator=gen, device="cuda", dtype=torch.uint8)
        a, b = table[pick[0].int()], table[pick[1].int()]
        flat[i:i + n] = a | (b << 4)
    return out


def _scales(gen, shape, typical):
    """Bytes E + 127 around 2^typical."""
    return (torch.randn(shape, generator=gen, device="cuda") * 0.7 + (127.5 + typical)).to(
        torch.uint8)


def _cache(gen, pages, heads, page, d):
    """Codes and scales of a whole cache: keys [pages][heads][page][dp / 2] bytes with scales
    [pages][heads][page][groups], values in blocks of four tokens, [pages][heads][page / 4]
    [dp / 8][4][4] bytes with scales [pages][heads][page / 4][groups][4].  dp: d in whole groups
    of 32."""
    g = -(-d // 32)
    return (_codes(gen, (pages, heads, page, 16 * g)),
            _codes(gen, (pages, heads, page // 4, 4 * g, 4, 4)),
            _scales(gen, (pages, heads, page, g), -1),
            _scales(gen, (pages, heads, page // 4, g, 4), -1))


def _pages(gen, need, spare=8):
    """The numbers of `need` pages of a cache with a few more, in the order a running server's
    free list gives them: any."""
    return torch.randperm(need + spare, generator=gen, device="cuda")[:need], need + spare


def _plan_inputs(case, seed):
    """(pool's table, lengths, free stack, count, entries' sequences, entries' new tokens)."""
    gen = _gen(seed)
    p, width, batch = case["page"], case["width"], case["batch"]
    lens = _lengths(case)
    rows = batch + case["spare"]
    r = random.Random(case["ragged"] + 1)
    at = r.sample(range(rows), batch)                     # the entries' sequences, in any order
    length = np.array([r.randint(0, case["past_hi"]) for _ in range(rows)], dtype=np.int32)
    for i, (n, m) in zip(at, lens):
        length[i] = m - n
    held = -(-length // p)
    taken = sum(-(-m // p) - -(-(m - n) // p) for n, m in lens)
    order, pages = _pages(gen, int(held.sum()) + taken + 40, 0)
    order = order.int()
    total = int(held.sum())
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    seen = torch.arange(width, device="cuda")[None, :] < torch.from_numpy(held).cuda()[:, None]
    table[seen] = order[:total]
    free = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    free[:pages - total] = order[total:]
    return (table, torch.from_numpy(length).cuda(), free,
            torch.tensor([pages - total], dtype=torch.int32, device="cuda"),
            torch.tensor(at, dtype=torch.int32, device="cuda"),
            torch.tensor([n for n, _ in lens], dtype=torch.int32, device="cuda"))


_SCALED = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=4.0),
           "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0),
           "ramp": dict(factor=16.0, original=4096, low=1.0, high=32.0)}
_BASE = {"none": 10000.0, "linear": 10000.0, "base": 10000.0, "bands": 500000.0, "ramp": 10000.0}


def _frequencies(case):
    """([radians a position] in 64 bits, amplitude)."""
    rot, kind = case["rot"], case["scaling"]
    base, s = _BASE[kind], _SCALED[kind]
    if kind == "base":
        base *= s["factor"] ** (rot / (rot - 2)) if rot > 2 else 1.0
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    amplitude = 1.0
    if kind == "linear":
        f = f / s["factor"]
    elif kind in ("bands", "ramp"):
        # turns over the original length: kept from `high` on, divided up to `low`; between, mixed
        # in proportion to the turns (bands) or to the place among the frequencies (ramp)
        turns = s["original"] * f / (2 * np.pi)
        if kind == "bands":
            keep = (turns - s["low"]) / (s["high"] - s["low"])
        else:
            def place(t):
                return rot * math.log(s["original"] / (t * 2 * math.pi)) / (2 * math.log(base))
            first = max(math.floor(place(s["high"])), 0)
            last = min(math.ceil(place(s["low"])), rot - 1)
            keep = 1 - (np.arange(rot // 2) - first) / max(last - first, 0.001)
            amplitude = 0.1 * math.log(s["factor"]) + 1.0
        keep = np.clip(keep, 0.0, 1.0)
        f = keep * f + (1 - keep) * f / s["factor"]
    return f, amplitude


def _rotary_inputs(case, seed):
    gen = _gen(seed)
    t, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["d"]
    x = _tokens(gen, t, (hq + 2 * hk) * d, _DT[case["dtype"]]).view(t, hq + 2 * hk, d)
    # sequences' stretches of positions up to `far`
    first = torch.randint(0, max(1, case["far"] - 1024), (t,), generator=gen, device="cuda")
    at = torch.arange(t, device="cuda")
    return x[:, :hq], x[:, hq:hq + hk], (first[at // 1024] + at % 1024).int()


def _cache_inputs(case, seed):
    gen = _gen(seed)
    t, r, h, d, p = case["tokens"], case["read"], case["heads"], case["d"], case["page"]
    dt = _DT[case["dtype"]]
    k = _tokens(gen, t, h * d, dt).reshape(t, h, d)
    v = _tokens(gen, t, h * d, dt).reshape(t, h, d)
    table, pages = _pages(gen, -(-r // p))
    at = torch.arange(r, device="cuda")
    slots = table[at // p] * p + at % p
    # the new tokens are the last of what is read back
    return k, v, slots, slots[r - t:].contiguous(), _cache(gen, pages, h, p, d)


def _attention_inputs(case, seed):
    gen = _gen(seed)
    h, d, p = case["kv_heads"], case["d"], case["page"]
    lens = _lengths(case)
    total = sum(n for n, _ in lens)
    q = torch.randn((total, h * case["group"], d), generator=gen, device="cuda") * 1.5
    per = [-(-m // p) for _, m in lens]
    order, pages = _pages(gen, sum(per))
    table = torch.zeros((len(lens), max(per)), dtype=torch.int32, device="cuda")
    first = 0
    for b, n in enumerate(per):
        table[b, :n] = order[first:first + n]
        first += n
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    return (q.to(_DT[case["dtype"]]), table,
            torch.tensor([m for _, m in lens], dtype=torch.int32, device="cuda"),
            torch.tensor(starts, dtype=torch.int32, device="cuda"), _cache(gen, pages, h, p, d))


def prepare(case, seed):
    kind = case["kind"]
    st = dict(case=case)
    if kind == "plan":
        st["table"], st["lengths"], st["free"], st["count"], st["seqs"], st["new"] = \
            _plan_inputs(case, seed)
        # a scheduler knows how many tokens its batch has at most; the last few are padding
        st["tokens"] = sum(n for n, _ in _lengths(case)) + 3
        st["before"] = st["lengths"][st["seqs"].long()].clone()
    elif kind == "rotary":
        st["q"], st["k"], st["positions"] = _rotary_inputs(case, seed)
        f, st["amplitude"] = _frequencies(case)
        st["freq"] = torch.from_numpy(f).cuda()
    elif kind == "cache":
        st["k"], st["v"], st["read"], st["write"], st["cache"] = _cache_inputs(case, seed)
    else:
        st["q"], st["table"], st["lens"], st["starts"], st["cache"] = _attention_inputs(case, seed)
        st["lengths"] = _lengths(case)                    # a scheduler knows them on the host too
    if own:
        from paper_2112_13896_amd import ops
        if kind == "plan":
            st["pool"] = ops.DevicePool(st["table"], st["lengths"], st["free"], st["count"],
                                        case["page"])
        elif kind == "rotary":
            st["rotary"] = ops.Rotary.make(case["rot"], base=_BASE[case["scaling"]],
                                           interleaved=case["interleaved"],
                                           scaling=case["scaling"], **_SCALED[case["scaling"]])
        else:
            st["cache"] = ops.PagedCache4(*st["cache"], d=case["d"])
        if kind == "attention":
            st["max_len"] = max(m for _, m in st["lengths"])
            st["ws"] = ops.paged_attention_workspace(st["q"], st["cache"], st["table"],
                                                     max_len=st["max_len"])
    return st


# ---------------------------------------------------------------- the operators
def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plain_plan, "rotary": _plain_rotary, "cache": _plain_cache,
            "attention": _plain_attention}[state["case"]["kind"]](state)


def _run_own(st):
    from paper_2112_13896_amd import ops
    kind = st["case"]["kind"]
    if kind == "plan":
        got = ops.plan_step(st["pool"], st["seqs"], st["new"], st["tokens"])
        ops.pool_truncate(st["pool"], st["seqs"], st["before"])
        return (*got, st["lengths"], st["free"], st["count"])
    if kind == "rotary":
        return ops.rotary(st["rotary"], st["positions"], st["q"], st["k"])
    if kind == "cache":
        ops.cache_write(st["cache"], st["k"], st["v"], st["write"])
        return ops.cache_read(st["cache"], st["read"], _DT[st["case"]["dtype"]])
    return ops.paged_attention(st["q"], st["cache"], st["table"], st["lens"], st["starts"],
                               window=st["case"]["window"], max_len=st["max_len"], ws=st["ws"])


def _plain_plan(st):
    """No entry is wrong and the pool has the pages: status is 0, 0."""
    case, pool, free = st["case"], st["table"], st["free"]
    p, width, cap = case["page"], case["width"], st["tokens"]
    seqs, new = st["seqs"].long(), st["new"].long()
    batch = seqs.numel()
    old = st["lengths"][seqs].long()
    held, full = (old + p - 1) // p, (old + new + p - 1) // p
    need = full - held
    before = torch.cumsum(need, 0) - need
    col = torch.arange(width, device="cuda")
    # new pages, the stack's top first
    fresh = st["count"].long() - 1 - (before[:, None] + col - held[:, None])
    is_new = (col >= held[:, None]) & (col < full[:, None])
    rows = torch.where(is_new, free[fresh.clamp(0, free.numel() - 1)], pool[seqs])
    pool[seqs] = rows
    table = torch.where(col < full[:, None], rows, -1)
    starts = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    starts[1:] = torch.cumsum(new, 0)
    st["lengths"][seqs] = (old + new).int()
    st["count"] -= need.sum().int()
    lens = (old + new).int()
    t = torch.arange(cap, device="cuda")
    entry = torch.searchsorted(starts[1:].long(), t, right=True)
    live = entry < batch
    e = entry.clamp(max=batch - 1)
    pos = torch.where(live, old[e] + t - starts[e], -1)
    slots = torch.where(live, table[e, (pos // p).clamp(min=0)].long() * p + pos % p, -1)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    # taken back: the pages past the old lengths go onto the stack, the last one first
    keep = (st["before"].long() + p - 1) // p
    drop = full - keep
    first = torch.cumsum(drop, 0) - drop
    total = drop.sum()
    gone = (col >= keep[:, None]) & (col < full[:, None])
    to = st["count"].long() + total - 1 - (first[:, None] + col - keep[:, None])
    # (one cell past the end takes what is not pushed)
    stack = torch.cat([free, free[:1]])
    stack[torch.where(gone, to, free.numel())] = rows
    free.copy_(stack[:-1])
    st["count"] += total.int()
    st["lengths"][seqs] = st["before"]
    return (table, lens, starts, slots, pos.int(), status, st["lengths"], free, st["count"])


def _plain_rotary(st):
    case, half = st["case"], st["case"]["rot"] // 2
    angle = st["positions"].double()[:, None] * st["freq"]
    cos = (torch.cos(angle) * st["amplitude"]).float()[:, None]
    sin = (torch.sin(angle) * st["amplitude"]).float()[:, None]
    out = []
    for x in (st["q"], st["k"]):
        y = x.float()
        if case["interleaved"]:
            a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        else:
            a, b = y[..., :half], y[..., half:2 * half]
        u, v = a * cos - b * sin, b * cos + a * sin
        if case["interleaved"]:
            z = torch.stack((u, v), dim=-1).flatten(-2)
        else:
            z = torch.cat((u, v), dim=-1)
        out.append(torch.cat((z, y[..., 2 * half:]), dim=-1).to(x.dtype))
    return tuple(out)


def _plain_values(codes):
    """Bytes [..., n] -> the codes' values [..., 2 n], low half first."""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).int()
    m, e = (c & 1).float(), (c >> 1 & 3).float()
    v = torch.where(e > 0, (1 + 0.5 * m) * torch.exp2(e - 1), 0.5 * m)
    return torch.where(c >= 8, -v, v)


def _plain_scales(s):
    return torch.where(s == 255, math.nan, torch.ldexp(torch.ones((), device="cuda"),
                                                       s.int() - 127))


def _plain_quantise(x):
    """(bytes of codes, scale bytes) of rows [..., d]."""
    d = x.shape[-1]
    g = -(-d // 32)
    x = torch.nn.functional.pad(x.float(), (0, 32 * g - d)).unflatten(-1, (g, 32))
    top = x.abs().amax(dim=-1)
    bad = ~torch.isfinite(top).all(dim=-1, keepdim=True)
    f, e = torch.frexp(top)                               # top = f * 2^e, f in [0.5, 1)
    e = torch.where(top == 0, -60, (e - 2 - (f <= 0.875).int()).clamp(-60, 60))
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for edge, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                     (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)
    code += 8 * torch.signbit(y).to(torch.uint8)
    code = torch.where(bad[..., None], 0, code).flatten(-2)
    scale = torch.where(bad, 255, e + 127).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _plain_cache(st):
    kc, vc, ks, vs = st["cache"]
    case = st["case"]
    p, d = case["page"], case["d"]
    page, off = st["write"] // p, st["write"] % p
    c, s = _plain_quantise(st["k"])
    kc[page, :, off], ks[page, :, off] = c, s
    c, s = _plain_quantise(st["v"])
    vc[page, :, off // 4, :, off % 4] = c.unflatten(-1, (-1, 4))
    vs[page, :, off // 4, :, off % 4] = s
    page, off = st["read"] // p, st["read"] % p
    out = []
    vals = vc[page, :, off // 4, :, off % 4].flatten(-2)
    for c, s in ((kc[page, :, off], ks[page, :, off]), (vals, vs[page, :, off // 4, :, off % 4])):
        y = _plain_values(c).unflatten(-1, (-1, 32)) * _plain_scales(s)[..., None]
        out.append(y.flatten(-2)[..., :d].to(_DT[case["dtype"]]))
    return tuple(out)


def _plain_attention(st):
    case = st["case"]
    kc, vc, ks, vs = st["cache"]
    h, g, d, p, win = case["kv_heads"], case["group"], case["d"], case["page"], case["window"]
    out = torch.empty_like(st["q"])
    first = 0
    for b, (n, m) in enumerate(st["lengths"]):
        lo = max(0, m - n - win + 1) // p * p if win else 0
        pages = st["table"][b, lo // p:-(-m // p)].long()
        keys = _plain_values(kc[pages]).unflatten(-1, (-1, 32))
        keys = keys * _plain_scales(ks[pages])[..., None]
        keys = keys.flatten(-2).transpose(0, 1).reshape(h, len(pages) * p, -1)
        # values: [page][head][block][8 channels][token] -> [page][head][block][token][channels]
        vals = _plain_values(vc[pages].transpose(-3, -2).flatten(-2))
        vals = vals.unflatten(-1, (-1, 32)) * _plain_scales(vs[pages].transpose(-2, -1))[..., None]
        vals = vals.flatten(-2).transpose(0, 1).reshape(h, len(pages) * p, -1)
        keys, vals = keys[:, :m - lo, :d], vals[:, :m - lo, :d]
        at = torch.arange(m - n, m, device="cuda")[:, None]
        j = torch.arange(lo, m, device="cuda")[None, :]
        seen = j <= at
        if win:
            seen = seen & (j > at - win)
        q = st["q"][first:first + n].float().reshape(n, h, g, d).permute(1, 2, 0, 3)
        some = max(1, min(h, (1 << 28) // max(1, g * n * (m - lo))))   # heads at a time
        for a in range(0, h, some):
            s = q[a:a + some].reshape(-1, g * n, d) @ keys[a:a + some].transpose(1, 2).contiguous()
            s = (s * (1.0 / math.sqrt(d))).reshape(-1, g, n, m - lo)
            s = torch.where(seen, s, -math.inf)
            e = torch.exp(s - s.amax(dim=-1, keepdim=True))
            e = e / e.sum(dim=-1, keepdim=True)
            o = e.reshape(-1, g * n, m - lo) @ vals[a:a + some].contiguous()
            o = o.reshape(-1, g, n, d)
            out[first:first + n, a * g:(a + o.shape[0]) * g] = \
                o.permute(2, 0, 1, 3).reshape(n, -1, d).to(out.dtype)
        first += n
    return out


# ---------------------------------------------------------------- costs
def work(case):
    """Every input and output once; of a cache, the tokens that the call uses; of a pool, the
    entries' pages.  2 operations for each product of a sum; the softmax is not counted."""
    kind = case["kind"]
    if kind == "plan":
        p, lens = case["page"], _lengths(case)
        held = sum(-(-(m - n) // p) for n, m in lens)
        taken = sum(-(-m // p) for _, m in lens) - held
        tokens, batch = sum(n for n, _ in lens) + 3, case["batch"]
        # pages read and written, those taken back once more; lengths and entries; tokens' outputs
        return dict(bytes=4 * (held + 3 * taken) + 4 * batch * case["width"] + 28 * batch
                    + 12 * tokens, flops=0)
    if kind == "rotary":
        x = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return dict(bytes=2 * x * case["d"] * _SIZE[case["dtype"]] + 4 * case["tokens"],
                    flops=3 * x * case["rot"])
    if kind == "cache":
        t, r, h, d = case["tokens"], case["read"], case["heads"], case["d"]
        e, held = _SIZE[case["dtype"]], d / 2 + -(-d // 32)
        return dict(bytes=int(2 * h * (t * (d * e + held) + r * (held + d * e))) + 8 * (t + r),
                    flops=2 * 2 * (t + r) * h * d)
    h, d, win = case["kv_heads"], case["d"], case["window"]
    pairs = tokens = rows = 0
    for n, m in _lengths(case):
        lo, hi = m - n + 1, m                             # keys seen by the first and last new one
        cap = min(hi, win) if win else hi
        below = max(0, min(hi, cap) - lo + 1)             # those that the window does not cut
        pairs += below * (2 * lo + below - 1) // 2 + (n - below) * cap
        tokens += min(m, n + win - 1) if win else m
        rows += n
    return dict(bytes=int(2 * tokens * h * (d / 2 + -(-d // 32)))
                + 2 * rows * h * case["group"] * d * _SIZE[case["dtype"]],
                flops=4 * d * h * case["group"] * pairs)


# ---------------------------------------------------------------- 64 bits
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plan64(case, seed):
    table, length, free, count, seqs, new = (t.cpu().numpy() for t in _plan_inputs(case, seed))
    p, width = case["page"], case["width"]
    lengths, stack = length.copy(), list(free[:count[0]])
    n_entries, cap = len(seqs), int(new.sum()) + 3
    out = np.full((n_entries, width), -1, dtype=np.int32)
    lens, starts = np.zeros(n_entries, np.int32), np.zeros(n_entries + 1, np.int32)
    slots, at = np.full(cap, -1, np.int64), np.full(cap, -1, np.int32)
    t = 0
    for i, (s, n) in enumerate(zip(seqs.tolist(), new.tolist())):
        held = -(-int(length[s]) // p)
        out[i, :held] = table[s, :held]
        lens[i] = length[s] + n
        for x in range(held, -(-int(lens[i]) // p)):
            out[i, x] = stack.pop()
        pos = np.arange(length[s], lens[i], dtype=np.int64)
        at[t:t + n] = pos
        slots[t:t + n] = out[i, pos // p].astype(np.int64) * p + pos % p
        t += n
        starts[i + 1] = t
    return tuple(torch.from_numpy(a) for a in (out, lens, starts, slots, at,
                                               np.zeros(2, np.int32), lengths, free, count))


def _grid64(x):
    """The values that the 4-bit codes of rows [rows][d] stand for."""
    x = x.double()
    res = torch.empty_like(x)
    points = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[-1], 32):
        part = x[..., c:c + 32]
        top = part.abs().max(dim=-1, keepdim=True).values
        e = torch.ceil(torch.log2(top / 7).clamp(-70, 70))
        e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, torch.where(top > 7 * torch.exp2(e),
                                                                         e + 1, e))
        s = torch.exp2(e.clamp(-60, 60))
        y = (part.abs() / s).clamp(max=6.0)
        dist = (y[..., None] - points).abs()
        # of two equally near codes the even one
        dist = dist + 1e-12 * (torch.arange(8, device=x.device) % 2)
        res[..., c:c + 32] = torch.copysign(points[dist.argmin(dim=-1)] * s, part)
    return res


def _codes64(byte):
    lut = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=torch.float64, device=byte.device)
    both = torch.empty(byte.shape[:-1] + (2 * byte.shape[-1],), dtype=torch.float64,
                       device=byte.device)
    both[..., 0::2] = lut[(byte % 16).int()]
    both[..., 1::2] = lut[(byte // 16).int()]
    return both


def _held64(cache, value, page, off, head, d):
    """Keys or values of the positions (page, offset) of one head, [positions][d]."""
    if value:
        code = cache[1][page, head, off // 4, :, off % 4].reshape(len(page), -1)
        byte = cache[3][page, head, off // 4, :, off % 4]
    else:
        code, byte = cache[0][page, head, off], cache[2][page, head, off]
    scale = torch.exp2(byte.double() - 127).repeat_interleave(32, dim=1)
    return (_codes64(code) * scale)[:, :d]


def exact(case, seed):
    if case["kind"] == "plan":
        return _plan64(case, seed)
    if case["kind"] == "rotary":
        q, k, positions = _rotary_inputs(case, seed)
        f, amplitude = _frequencies(case)
        turn = torch.polar(torch.full((), amplitude, dtype=torch.float64, device="cuda"),
                           positions.double()[:, None] * torch.from_numpy(f).cuda())[:, None]
        res, rot = [], case["rot"]
        for x in (q, k):
            y = x.double()
            i = torch.arange(rot, device="cuda")
            i = i.view(-1, 2).t() if case["interleaved"] else i.view(2, -1)
            z = torch.complex(y[..., i[0]], y[..., i[1]]) * turn
            y[..., i[0]], y[..., i[1]] = z.real, z.imag
            res.append(y)
        return tuple(res)
    if case["kind"] == "cache":
        k, v, read, _, cache = _cache_inputs(case, seed)
        p, t, h, d = case["page"], case["tokens"], case["heads"], case["d"]
        res = []
        for value, x in ((False, k), (True, v)):
            old = torch.stack([_held64(cache, value, read // p, read % p, i, d) for i in range(h)],
                              dim=1)
            for at in range(0, t, 2048):
                old[old.shape[0] - t + at:][:2048] = _grid64(x[at:at + 2048])
            res.append(old)
        return tuple(res)
    q, table, _, _, cache = _attention_inputs(case, seed)
    lens = _lengths(case)
    g, d, p, win = case["group"], case["d"], case["page"], case["window"]
    if sum(n * m for n, m in lens) * case["kv_heads"] * g * d > 3e12:
        return None
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, m) in enumerate(lens):
        pos = torch.arange(m, device="cuda")
        page, off = table[b].long()[pos // p], pos % p
        new = torch.arange(n, device="cuda") + (m - n)
        hidden = pos[None, :] > new[:, None]
        if win:
            hidden |= pos[None, :] <= new[:, None] - win
        for kv in range(case["kv_heads"]):
            key = _held64(cache, False, page, off, kv, d).t().contiguous()
            val = _held64(cache, True, page, off, kv, d).contiguous()
            for head in range(kv * g, (kv + 1) * g):
                logit = torch.mm(q[first:first + n, head].double(), key) / math.sqrt(d)
                logit = logit.masked_fill_(hidden, -math.inf)
                out[first:first + n, head] = torch.mm(torch.softmax(logit, dim=1), val)
        first += n
    return out
