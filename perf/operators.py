"""Block tables built on the GPU and sparse decode attention over a block-paged cache, as timed cases.

Four kinds of calls, in the order a serving program makes them:

  reserve   paged_reserve() of a step's new tokens - block table entries and the slot map from the lengths - and paged_trim()
            back to the lengths before, as a step whose drafted tokens are all rejected makes them
  write     paged_write(): new key and value rows, views of a fused projection's output, into the pages by their slots
  bounds    paged_bounds(): per channel the least and largest key of every block that new tokens touched, and its degrees' sum
  sparse    paged_select() and paged_sparse_decode_attn(): the blocks of the largest upper bound of softmax mass per
            (sequence, KV head), and decode attention over those alone

`own` chooses between the plain form of each and the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_IN_USE = 2**31 - 1             # a free list's mark of a block that is taken; -1: free
_SCRATCH = 1 << 25              # the workspace a program keeps for its select and attention calls
_MOST = 1 << 31                 # bytes of the largest key pool


# ---- the listed cases -----------------------------------------------------------------------------
def listed():
    return [
        # a decode step of 64 requests, one token each: nothing but latency
        _reserve("reserve_step_64", batch=64, tokens=8192, new=1),
        # a wave of prompts of all lengths, and idle rows
        _reserve("reserve_prompts_33x8k", batch=33, tokens=1000, new=8192, block=32),
        # many short requests drafting up to seven tokens, the pool short of what they ask for: the later ones are refused
        _reserve("reserve_tight_1000", batch=1000, tokens=700, new=7, short=True),
        # the new rows of a decode step
        _write("write_step_64", rows=64),
        # prompts packed one behind the other, with padding rows behind the last
        _write("write_prompts_50k", rows=50021, pad=91),
        # a decode step's last blocks
        _bounds("bounds_step_64", batch=64, tokens=8192, step=True),
        # whole prompts, with the degrees a compressed cache has
        _bounds("bounds_prompts_8x32k", batch=8, tokens=32768),
        # one request with a short context: latency
        _sparse("sparse_short_1x2k", batch=1, tokens=2050, select=32),
        # serving: 16 requests of different lengths, a sixteenth of the cache read
        _sparse("sparse_serving_16x32k", batch=16, tokens=32768, select=128),
        # one request with an extreme context
        _sparse("sparse_long_1x1m", batch=1, tokens=1 << 20, select=256, degrees=False),
        # fp32 caches, odd lengths, small heads
        _sparse("sparse_f32_5x9k", batch=5, tokens=9001, select=48, heads=4, group=2, dim=64, dtype="f32", block=32),
        # many requests on large blocks, eight query heads per KV head, no degrees
        _sparse("sparse_wide_61x8k", batch=61, tokens=8192, select=24, group=8, block=64, degrees=False),
    ]


def _reserve(name, batch, tokens, new, block=16, short=False):
    return dict(name=name, kind="reserve", batch=batch, tokens=tokens, new=new, block=block, short=short)


def _write(name, rows, pad=0, heads=8, group=4, dim=128, dtype="bf16", block=16, degrees=True):
    return dict(name=name, kind="write", rows=rows, pad=pad, heads=heads, group=group, dim=dim, dtype=dtype, block=block,
                degrees=degrees)


def _bounds(name, batch, tokens, step=False, heads=8, dim=128, dtype="bf16", block=16, degrees=True):
    return dict(name=name, kind="bounds", batch=batch, tokens=tokens, step=step, heads=heads, dim=dim, dtype=dtype, block=block,
                degrees=degrees)


def _sparse(name, batch, tokens, select, heads=8, group=4, dim=128, dtype="bf16", block=16, degrees=True):
    return dict(name=name, kind="sparse", batch=batch, tokens=tokens, select=select, heads=heads, group=group, dim=dim,
                dtype=dtype, block=block, degrees=degrees)


# ---- more cases of the same ranges ----------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("reserve", "write", "bounds", "sparse", "sparse", "sparse"))
    block = rng.choice((8, 16, 16, 32, 64))
    if kind == "reserve":
        batch = _log(rng, 1, 1500)
        new = 1 if rng.random() < 0.4 else _log(rng, 1, max(2, 200000 // batch))
        case = _reserve("", batch, tokens=_log(rng, 1, max(2, min(32768, (1 << 21) // batch))), new=min(new, 65536), block=block,
                        short=rng.random() < 0.2)
    else:
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        heads, dim = rng.choice((1, 2, 4, 8, 8)), rng.choice((64, 128, 128) + ((32,) if dtype == "f32" else ()))
        row = heads * dim * (4 if dtype == "f32" else 2)
        shape = dict(heads=heads, dim=dim, dtype=dtype, block=block, degrees=rng.random() < 0.7)
        if kind == "write":
            case = _write("", rows=_log(rng, 1, min(50000, (1 << 27) // row)), pad=rng.choice((0, 0, 7, 100)),
                          group=rng.choice((1, 2, 4, 8)), **shape)
        else:
            batch = _log(rng, 1, 64)
            most = (_MOST if kind == "sparse" else _MOST // 4) // (row * batch)
            tokens = _log(rng, 16, max(17, min(1 << 20 if batch < 3 else 1 << 17, most)))
            if kind == "bounds":
                case = _bounds("", batch, tokens, step=rng.random() < 0.4, **shape)
            else:
                case = _sparse("", batch, tokens, select=min(_log(rng, 4, 256), max(4, 6144 // block)), group=rng.choice((1, 2, 4, 4, 8)),
                               **shape)
    del case["name"]
    return case


# ---- what a program has in hand before the call ---------------------------------------------------
def _spread(n, lo, hi, gen):
    """n whole numbers spread evenly over [lo, hi], in an order that the seed gives."""
    v = np.linspace(lo, hi, n).round().astype(np.int64) if n > 1 else np.array([hi])
    return torch.from_numpy(v)[torch.randperm(n, generator=gen)]


def _lens(case, gen):
    return _spread(case["batch"], max(case["tokens"] // 2, 1), case["tokens"], gen)


def _tables(lens, block, max_blocks, gen, spare=0):
    """(table, n_blocks, order): blocks of a shuffled pool dealt to the rows, -1 behind them; order: the pool's shuffle."""
    need = (lens + block - 1) // block
    n_blocks = int(need.sum()) + spare
    order = torch.randperm(n_blocks, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max_blocks), -1, dtype=torch.int32)
    table[torch.arange(max_blocks)[None] < need[:, None]] = order[:int(need.sum())]
    return table, n_blocks, order


def _int(x):
    return x.to(torch.int32).to(DEV)


def _pool(gen, n_blocks, heads, block, dim, dtype):
    """Keys of a pool: the tokens of a block around a mean of their own, one channel in 32 ten times as loud."""
    K = torch.empty((n_blocks, heads, block, dim), dtype=_DT[dtype], device=DEV).normal_(generator=gen).mul_(0.45)
    loud = torch.ones((heads, dim), device=DEV)
    loud[:, torch.randperm(dim, generator=gen, device=DEV)[:dim // 32]] = 10.0
    mean = torch.empty((n_blocks, heads, 1, dim), device=DEV).normal_(generator=gen).mul_(0.9)
    return K.add_(mean.to(K.dtype)).mul_(loud[:, None].to(K.dtype))


def _degrees(gen, shape):
    """Cluster sizes of a cache compressed to a quarter: 1 and up, four on average."""
    return 1 + torch.empty(shape, device=DEV).exponential_(1.0 / 3.5, generator=gen).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))
    return {"reserve": _prepare_reserve, "write": _prepare_write, "bounds": _prepare_bounds,
            "sparse": _prepare_sparse}[case["kind"]](case, gen, host)


def _prepare_reserve(case, gen, host):
    batch, block = case["batch"], case["block"]
    lens = _spread(batch, 0, case["tokens"], host)
    new = _spread(batch, 0 if batch > 8 and case["new"] > 1 else 1, case["new"], host)
    # free blocks: enough for any order of these numbers, or too few for what is asked for on average
    spare = max(1, int(new.sum()) * 3 // (4 * block)) if case["short"] else batch + int(((new + block - 1) // block).sum())
    max_blocks = (case["tokens"] + case["new"] + block - 1) // block + 1
    table, n_blocks, order = _tables(lens, block, max_blocks, host, spare)
    used = n_blocks - spare
    free = torch.full((4 + 2 * n_blocks,), -1, dtype=torch.int32)
    free[:4] = 0
    free[0] = spare
    free[4:4 + spare] = order[used:]
    free[4 + n_blocks:][order[:used].long()] = _IN_USE
    slots = (int(new.sum()) + 127) // 128 * 128
    empty = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    return dict(kind="reserve", table=table.to(DEV), lens=_int(lens), before=_int(lens), new=_int(new), free=free.to(DEV), block=block,
                n_slots=slots, out=(empty(slots), empty(batch + 1), empty(batch)))


def _prepare_write(case, gen, host):
    rows, pad, heads, dim, block = case["rows"], case["pad"], case["heads"], case["dim"], case["block"]
    dt, q_heads = _DT[case["dtype"]], heads * case["group"]
    qkv = torch.empty((rows + pad, q_heads + 2 * heads, dim), dtype=dt, device=DEV).normal_(generator=gen)
    n_blocks = rows // block + 9
    order = torch.randperm(n_blocks, generator=host)
    t = torch.arange(rows) + 5                       # the first row continues a block
    slots = torch.cat([order[t // block] * block + t % block, torch.full((pad,), -1)])
    shape = (n_blocks, heads, block)
    K, V = (torch.zeros(shape + (dim,), dtype=dt, device=DEV) for _ in range(2))
    return dict(kind="write", k=qkv[:, q_heads:q_heads + heads], v=qkv[:, q_heads + heads:], slots=_int(slots), rows=rows, K=K, V=V,
                deg=torch.zeros(shape, dtype=torch.int32, device=DEV) if case["degrees"] else None)


def _prepare_bounds(case, gen, host):
    block, lens = case["block"], _lens(case, host)
    table, n_blocks, _ = _tables(lens, block, (case["tokens"] + block - 1) // block + 2, host, spare=3)
    K = _pool(gen, n_blocks, case["heads"], block, case["dim"], case["dtype"])
    out = (torch.zeros((n_blocks, case["heads"], 2, case["dim"]), dtype=K.dtype, device=DEV),
           torch.zeros((n_blocks, case["heads"]), dtype=torch.int32, device=DEV))
    return dict(kind="bounds", K=K, deg=_degrees(gen, K.shape[:3]) if case["degrees"] else None, table=table.to(DEV), lens=_int(lens),
                since=_int(lens - 1) if case["step"] else None, max_new=1 if case["step"] else case["tokens"], out=out)


def _prepare_sparse(case, gen, host):
    block, heads, dim, batch = case["block"], case["heads"], case["dim"], case["batch"]
    lens = _lens(case, host)
    table, n_blocks, _ = _tables(lens, block, (case["tokens"] + block - 1) // block + 2, host, spare=3)
    K = _pool(gen, n_blocks, heads, block, dim, case["dtype"])
    V = torch.empty_like(K).normal_(generator=gen)
    deg = _degrees(gen, K.shape[:3]) if case["degrees"] else None
    bounds = torch.stack([K.amin(2), K.amax(2)], 2)
    mass = deg.sum(2, dtype=torch.int32) if case["degrees"] else torch.full((n_blocks, heads), block, dtype=torch.int32, device=DEV)
    q = torch.empty((batch, heads * case["group"], dim), device=DEV).normal_(generator=gen).to(K.dtype)
    out = (torch.zeros((batch, heads, case["select"]), dtype=torch.int32, device=DEV),
           torch.zeros((batch, heads), dtype=torch.int32, device=DEV))
    return dict(kind="sparse", q=q, K=K, V=V, deg=deg, bounds=bounds, mass=mass, table=table.to(DEV), lens=_int(lens),
                max_len=case["tokens"], n_select=case["select"], block=block, out=out, o=torch.zeros_like(q),
                ws=torch.zeros(_SCRATCH, dtype=torch.uint8, device=DEV), ws_attn=torch.zeros(_SCRATCH, dtype=torch.uint8, device=DEV))


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if kind == "reserve":
        return _own_reserve(s) if own else _plain_reserve(s)
    if kind == "write":
        return _own_write(s) if own else _plain_write(s)
    if kind == "bounds":
        return _own_bounds(s) if own else _plain_bounds(s)
    return _own_sparse(s) if own else _plain_sparse(s)


def _own_reserve(s):
    import paper_2506_11418_amd as ckv
    slots, starts, granted = ckv.paged_reserve(s["table"], s["lens"], s["new"], s["free"], s["block"], s["n_slots"], out=s["out"])
    ckv.paged_trim(s["table"], s["lens"], s["before"], s["free"], s["block"])
    return slots, starts, granted, s["table"], s["lens"], s["free"]


def _own_write(s):
    import paper_2506_11418_amd as ckv
    ckv.paged_write(s["k"], s["v"], s["slots"], s["K"], s["V"], s["deg"])
    return [s["K"], s["V"]] + ([] if s["deg"] is None else [s["deg"]])


def _own_bounds(s):
    import paper_2506_11418_amd as ckv
    return ckv.paged_bounds(s["K"], s["deg"], s["table"], s["lens"], s["max_new"], since=s["since"], out=s["out"])


def _own_sparse(s):
    import paper_2506_11418_amd as ckv
    sel, sel_lens = ckv.paged_select(s["q"], s["bounds"], s["mass"], s["table"], s["lens"], s["max_len"], s["n_select"], s["block"],
                                     n_sink=1, n_recent=1, out=s["out"], workspace=s["ws"])
    o = ckv.paged_sparse_decode_attn(s["q"], s["K"], s["V"], s["deg"], sel, sel_lens, out=s["o"], workspace=s["ws_attn"])
    return sel, sel_lens, o


def _plain_reserve(s):
    table, lens, free, block, n_slots = s["table"], s["lens"], s["free"], s["block"], s["n_slots"]
    n_blocks, width = (len(free) - 4) // 2, table.shape[1]
    stack, marks, count = free[4:4 + n_blocks], free[4 + n_blocks:], free[0].long()
    L, new = lens.long(), s["new"].long().clamp(min=0)
    ends = new.cumsum(0)
    fits = (L >= 0) & (L + new <= width * block) & (ends <= n_slots)
    first = (L + block - 1) // block
    need = torch.where(fits, (L + new + block - 1) // block - first, 0)
    granted = fits & ((need == 0) | (need.cumsum(0) <= count))
    take = torch.where(granted, need, 0)
    base = take.cumsum(0) - take
    k = torch.arange(width, device=DEV)[None] - first[:, None]
    fresh = (k >= 0) & (k < take[:, None])
    table.copy_(torch.where(fresh, stack[(count - 1 - base[:, None] - k).clamp(0, n_blocks - 1)], table))
    at = torch.arange(n_blocks, device=DEV)
    marks.scatter_reduce_(0, stack.long().clamp(min=0), torch.where((at < count) & (at >= count - take.sum()), _IN_USE, -1).to(torch.int32),
                          "amax")
    j = torch.arange(n_slots, device=DEV)
    b = torch.searchsorted(ends, j, right=True).clamp(max=len(L) - 1)
    t = (L[b] + j - (ends - new)[b]).clamp(0, width * block - 1)
    blk = table[b, t // block].long()
    inside = (j < ends[-1]) & granted[b] & (blk >= 0) & (blk < n_blocks)
    slots = torch.where(inside, blk * block + t % block, -1).to(torch.int32)
    starts = torch.cat([ends.new_zeros(1), ends]).clamp(max=n_slots).to(torch.int32)
    grown = torch.where(granted, L + new, L)
    lens.copy_(grown)
    left = count - take.sum()
    free[0] = left
    # and back to the lengths before: entries behind them return to the stack, the last of the last row first
    back = s["before"].long()
    cut = (back >= 0) & (back < grown)
    col = torch.arange(width, device=DEV)[None]
    gone = cut[:, None] & (col >= ((back + block - 1) // block)[:, None]) & (col < ((grown + block - 1) // block)[:, None])
    ids, ok = table.flatten().flip(0).long(), gone.flatten().flip(0)
    ok = ok & (ids >= 0) & (ids < n_blocks) & (marks[ids.clamp(0, n_blocks - 1)] == _IN_USE)
    place = torch.where(ok, left + ok.cumsum(0) - 1, n_blocks)
    stack.copy_(torch.cat([stack, stack[:1]]).scatter_(0, place, ids.to(torch.int32))[:n_blocks])
    marks.scatter_reduce_(0, ids.clamp(0, n_blocks - 1), torch.where(ok, -1, _IN_USE).to(torch.int32), "amin")
    table.copy_(torch.where(gone, -1, table))
    lens.copy_(torch.where(cut, back, grown))
    free[0] = left + ok.sum()
    return slots, starts, granted.to(torch.int32), table, lens, free


def _plain_write(s):
    K, V, deg = s["K"], s["V"], s["deg"]
    block = K.shape[2]
    slot = s["slots"][:s["rows"]].long()                              # (what is behind is padding)
    K[slot // block, :, slot % block] = s["k"][:s["rows"]]
    V[slot // block, :, slot % block] = s["v"][:s["rows"]]
    if deg is None:
        return [K, V]
    deg[slot // block, :, slot % block] = 1
    return [K, V, deg]


def _touched(s, since):
    """Which table columns hold tokens [since, lens) of their row, and how many tokens of those blocks count."""
    block, table, lens = s["K"].shape[2], s["table"], s["lens"].long()[:, None]
    col = torch.arange(table.shape[1], device=DEV)[None]
    hit = (col >= since // block) & (col * block < lens) & (table >= 0)
    return hit, (lens - col * block).clamp(0, block)


def _plain_bounds(s):
    K, deg, (bounds, mass) = s["K"], s["deg"], s["out"]
    hit, n = _touched(s, 0 if s["since"] is None else s["since"].long()[:, None])
    blk, n = s["table"][hit].long(), n[hit]
    k = K[blk]
    counted = (torch.arange(K.shape[2], device=DEV)[None] < n[:, None])[:, None, :]
    if deg is not None:
        counted = counted & (deg[blk] > 0)
    bounds[blk, :, 0] = k.masked_fill(~counted[..., None], math.inf).amin(2)
    bounds[blk, :, 1] = k.masked_fill(~counted[..., None], -math.inf).amax(2)
    mass[blk] = (counted.expand(-1, K.shape[1], -1) if deg is None else torch.where(counted, deg[blk], 0)).sum(2, dtype=torch.int32)
    return bounds, mass


def _scale(dim):
    return float(np.float32(1.0) / np.sqrt(np.float32(dim)))


def _plain_sparse(s):
    q, table, lens, block, n_select = s["q"], s["table"], s["lens"].long(), s["block"], s["n_select"]
    (batch, q_heads, dim), (n_pool, heads) = q.shape, s["mass"].shape
    group, width, scale = q_heads // heads, min(table.shape[1], -(-s["max_len"] // block)), _scale(dim)
    blk = table[:, :width].long()
    h = torch.arange(heads, device=DEV)[None, :, None]
    at = blk.clamp(min=0)[:, None]                                    # [batch, 1, width]
    # the score in 64 bits: its order decides, and neighbours at the cut are close
    b = s["bounds"][at, h].double()                                   # [batch, heads, width, 2, dim]
    qd = q.double().view(batch, heads, group, dim)
    dots = torch.matmul(torch.cat([qd.clamp(max=0), qd.clamp(min=0)], 3), b.view(batch, heads, width, 2 * dim).transpose(2, 3))
    m = s["mass"][at, h]
    score = (dots.amax(2) * scale + torch.log(m.double())).float()    # [batch, heads, width]
    col = torch.arange(width, device=DEV)[None, None]
    last = ((lens + block - 1) // block)[:, None, None]
    score = torch.where((m > 0) & (blk >= 0)[:, None], score, -math.inf)
    score = torch.where((col < 1) | (col >= last - 1), math.inf, score)
    score = torch.where(col < last, score, -math.inf)
    chosen = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :n_select]
    chosen = torch.where(chosen < last, chosen, width).sort(2).values
    pos = torch.full((batch, heads, n_select), width, device=DEV)
    pos[:, :, :chosen.shape[2]] = chosen
    some = pos < last
    ids = torch.where(some, blk[:, None].expand(-1, heads, -1).gather(2, pos.clamp(max=width - 1)), -1)
    sel = torch.where(ids >= 0, ids * heads + h, -1).to(torch.int32)
    tokens = torch.where(some, (lens[:, None, None] - pos * block).clamp(0, block), 0)
    # attention over the blocks chosen
    at = ids.clamp(min=0)
    k, v = (p[at, h].float().view(batch, heads, n_select * block, dim) for p in (s["K"], s["V"]))
    logits = torch.matmul(q.float().view(batch, heads, group, dim), k.transpose(2, 3)) * scale
    if s["deg"] is not None:
        logits = logits + torch.log(s["deg"][at, h].float()).view(batch, heads, 1, -1)
    inside = (torch.arange(block, device=DEV) < tokens[..., None]) & (ids >= 0)[..., None]
    logits = logits.masked_fill(~inside.view(batch, heads, 1, -1), -math.inf)
    w = torch.exp(logits - logits.amax(3, keepdim=True))
    o = torch.matmul(w, v) / w.sum(3, keepdim=True)
    return sel, tokens.sum(2).to(torch.int32), o.view(batch, q_heads, dim).to(q.dtype)


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    block = case["block"]
    up = lambda n: -(-n // block)
    if case["kind"] == "reserve":
        tokens = case["batch"] * case["new"] * (0.5 if case["new"] > 1 else 1)
        # lengths and new tokens read, lengths, flags and starts written, twice for lengths; slots; stack, table and mark of a block
        return dict(bytes=28 * case["batch"] + 4 * tokens + 24 * max(tokens / block, 1), flops=0)
    row = case["heads"] * case["dim"] * (4 if case["dtype"] == "f32" else 2)
    per_token = 4 * case["heads"] if case["degrees"] else 0
    if case["kind"] == "write":
        return dict(bytes=case["rows"] * (4 * row + per_token + 4) + 4 * case["pad"], flops=0)
    tokens = case["batch"] * case["tokens"] * 0.75 if case["batch"] > 1 else case["tokens"]
    if case["kind"] == "bounds":
        if case["step"]:
            tokens = case["batch"] * block / 2
        blocks = tokens / block
        return dict(bytes=tokens * (row + per_token) + blocks * (2 * row + 4 * case["heads"] + 4), flops=2 * tokens * row)
    blocks, group = tokens / block, case["group"]
    chosen = min(case["select"] * block * case["batch"], tokens)
    heads = case["heads"]
    answer = case["batch"] * (2 * group * row + 4 * heads * case["select"])
    return dict(bytes=blocks * (2 * row + 4 * heads + 4) + chosen * (2 * row + per_token) + answer,
                flops=4 * group * heads * case["dim"] * (blocks + chosen))


# ---- the definitions in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "reserve":
        return None
    s = prepare(case, seed)
    return {"write": _exact_write, "bounds": _exact_bounds, "sparse": _exact_sparse}[s["kind"]](s)


def _exact_write(s):
    """Row r of the pool seen as one token after the other is what the slot map says, or what it was."""
    K, V, deg = s["K"], s["V"], s["deg"]
    n_blocks, heads, block, dim = K.shape
    source = torch.full((n_blocks * block + 1,), -1, dtype=torch.int64, device=DEV)
    source[s["slots"].long()] = torch.arange(len(s["slots"]), device=DEV)     # (padding rows: the last entry)
    source = source[:-1].view(n_blocks, block)
    outs = []
    for pool, new in ((K, s["k"]), (V, s["v"])):
        rows = torch.where((source >= 0)[..., None, None], new[source.clamp(min=0)], pool.permute(0, 2, 1, 3))
        outs.append(rows.permute(0, 2, 1, 3).double())
    return outs + ([] if deg is None else [None])


def _exact_bounds(s):
    K, deg, bounds = s["K"], s["deg"], s["out"][0].double()
    block = K.shape[2]
    for b, n in enumerate(s["lens"].tolist()):
        lo = 0 if s["since"] is None else int(s["since"][b]) // block
        hi = -(-n // block)
        ids = s["table"][b, lo:hi].long()
        k = K[ids].double()                                        # [blocks, heads, block, dim]
        tail = torch.arange(lo * block, hi * block, device=DEV).view(-1, 1, block, 1) >= n
        skip = tail if deg is None else tail | (deg[ids] < 1)[..., None]
        bounds[ids, :, 0] = torch.where(skip, math.inf, k).min(2).values
        bounds[ids, :, 1] = torch.where(skip, -math.inf, k).max(2).values
    return bounds, None


def _exact_sparse(s):
    q, (n_pool, heads), block = s["q"].double(), s["mass"].shape, s["block"]
    batch, q_heads, dim = q.shape
    group, scale, o = q_heads // heads, _scale(dim), torch.zeros_like(q)
    for b, n in enumerate(s["lens"].tolist()):
        ids = s["table"][b, :-(-n // block)].long()
        for h in range(heads):
            mine = q[b, h * group:(h + 1) * group]
            bound = s["bounds"][ids, h].double()
            best = torch.stack([torch.maximum(x * bound[:, 0], x * bound[:, 1]).sum(1) for x in mine]).max(0).values
            score = (best * scale + s["mass"][ids, h].double().log()).float()
            score[0] = score[-1] = math.inf
            keep = torch.sort(-score, stable=True).indices[:s["n_select"]].sort().values
            token = (keep[:, None] * block + torch.arange(block, device=DEV)).flatten()
            k, v = (p[ids[keep], h].reshape(-1, dim)[token < n].double() for p in (s["K"], s["V"]))
            x = mine @ k.T.contiguous() * scale
            if s["deg"] is not None:
                x = x + s["deg"][ids[keep], h].flatten()[token < n].double().log()
            o[b, h * group:(h + 1) * group] = torch.softmax(x, 1) @ v
    return None, None, o
