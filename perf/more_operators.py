"""Attention of new tokens over a block-paged cache, and pages forked, copied and compacted, as timed cases.

Three kinds of calls:

  chunk     paged_chunk_attn(): several new tokens of every sequence against its pages - prompts in pieces, a second turn on a
            compressed cache, drafted tokens to verify, single tokens among them; without the causal mask a decoder's tokens
            against an encoder's states
  fork      paged_fork() and paged_copy(): rows that continue a prompt get blocks of their own, and the prompt's pages are
            copied into them; then paged_trim() of the forked rows, as a search that drops its candidates makes it
  compact   a serving pool as requests come and go: half of the rows finish (paged_trim()), the others' highest blocks move into
            the lowest free ones (paged_compact() and paged_copy()), as many new rows of the same lengths arrive
            (paged_reserve()); then the same with the other half

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
_SCRATCH = 1 << 29              # the workspace a program keeps for its attention calls
_MOST = 1 << 31                 # bytes of the largest key pool


# ---- the listed cases -----------------------------------------------------------------------------
def listed():
    return [
        # one short request, a few new tokens: latency
        _chunk("chunk_short_1x33", batch=1, tokens=515, new=33),
        # drafted tokens, one to eight a request, verified against compressed caches
        _chunk("chunk_verify_16x8_32k", batch=16, tokens=32768, new=8, ragged=True),
        # a decode step that takes a piece of one request's prompt along: single tokens and one long row
        _chunk("chunk_mixed_40_16k", batch=40, tokens=16384, new=1999, mixed=True, pad=57),
        # a first prompt, nothing before it
        _chunk("chunk_prompt_1x16k", batch=1, tokens=0, new=16384, degrees=False),
        # second turns of 4 requests over what is left of the first
        _chunk("chunk_turn_4x2k_16k", batch=4, tokens=16384, new=2048, ragged=True),
        # fp32 caches, small heads, odd lengths
        _chunk("chunk_f32_3x301_2k", batch=3, tokens=2050, new=301, heads=4, group=2, dim=64, dtype="f32", block=32, ragged=True),
        # a decoder's tokens against an encoder's states: every one of them sees all
        _chunk("chunk_cross_9x700_1500", batch=9, tokens=1500, new=700, heads=12, group=1, dim=64, block=64, degrees=False, ragged=True,
               causal=False),
        # one prompt of a few blocks forked once: latency
        _fork("fork_short_1x500", sources=1, copies=1, tokens=500),
        # the best of eight continuations of a long prompt
        _fork("fork_best_of_8_16k", sources=1, copies=7, tokens=16384),
        # many prompts forked twice, free blocks for three quarters of them
        _fork("fork_tight_33x2x2k", sources=33, copies=2, tokens=2050, block=32, short=True),
        # a few short requests come and go: latency
        _compact("compact_small_6x500", pairs=3, tokens=500),
        # a serving pool
        _compact("compact_serving_64x8k", pairs=32, tokens=8192),
    ]


def _chunk(name, batch, tokens, new, heads=8, group=4, dim=128, dtype="bf16", block=16, degrees=True, ragged=False, mixed=False, pad=0,
           causal=True):
    return dict(name=name, kind="chunk", batch=batch, tokens=tokens, new=new, heads=heads, group=group, dim=dim, dtype=dtype, block=block,
                degrees=degrees, ragged=ragged, mixed=mixed, pad=pad, causal=causal)


def _fork(name, sources, copies, tokens, heads=8, dim=128, dtype="bf16", block=16, short=False):
    return dict(name=name, kind="fork", sources=sources, copies=copies, tokens=tokens, heads=heads, dim=dim, dtype=dtype, block=block,
                short=short)


def _compact(name, pairs, tokens, heads=8, dim=128, dtype="bf16", block=16):
    return dict(name=name, kind="compact", pairs=pairs, tokens=tokens, heads=heads, dim=dim, dtype=dtype, block=block)


# ---- more cases of the same ranges ----------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("chunk", "chunk", "chunk", "fork", "compact"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads, dim = rng.choice((1, 2, 4, 8, 8)), rng.choice((64, 128, 128) + ((32,) if dtype == "f32" else ()))
    block = rng.choice((8, 16, 16, 32, 64))
    row = heads * dim * (4 if dtype == "f32" else 2)
    shape = dict(heads=heads, dim=dim, dtype=dtype, block=block)
    if kind == "chunk":
        group, batch = rng.choice((1, 2, 4, 4, 8)), _log(rng, 1, 64)
        tokens = _log(rng, 16, max(17, min(65536, _MOST // (row * batch))))
        # as many new tokens as cost no more than the largest listed case (fp32: an eighth of it)
        most = (1 << 41) / (8 if dtype == "f32" else 1) / (4 * heads * group * dim)
        new = most / (batch * tokens)
        if new > tokens:
            new = math.sqrt(most / batch)
        new = _log(rng, 1, max(2, min(16384, int(new))))
        causal = rng.random() < 0.8
        case = _chunk("", batch, tokens, new, group=group, degrees=rng.random() < 0.7, ragged=rng.random() < 0.6, causal=causal,
                      mixed=batch > 2 and rng.random() < 0.2, pad=rng.choice((0, 0, 7, 100)), **shape)
    elif kind == "fork":
        sources, copies = _log(rng, 1, 40), _log(rng, 1, 8)
        tokens = _log(rng, 8, max(9, min(32768, (_MOST // 4) // (row * sources * (1 + copies)))))
        case = _fork("", sources, copies, tokens, short=rng.random() < 0.2, **shape)
    else:
        pairs = _log(rng, 1, 40)
        case = _compact("", pairs, tokens=_log(rng, 8, max(9, min(32768, (_MOST // 4) // (row * 2 * pairs)))), **shape)
    del case["name"]
    return case


# ---- what a program has in hand before the call ---------------------------------------------------
def _spread(n, lo, hi, gen):
    """n whole numbers spread evenly over [lo, hi], in an order that the seed gives."""
    v = np.linspace(lo, hi, n).round().astype(np.int64) if n > 1 else np.array([hi])
    return torch.from_numpy(v)[torch.randperm(n, generator=gen)]


def _int(x):
    return torch.as_tensor(x).to(torch.int32).to(DEV)


def _up(n, block):
    return -(-n // block)


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
    return {"chunk": _prepare_chunk, "fork": _prepare_fork, "compact": _prepare_compact}[case["kind"]](case, gen, host)


def _chunk_lens(case, host):
    """(tokens before, new tokens) of every sequence."""
    batch, new = case["batch"], case["new"]
    before = _spread(batch, case["tokens"] // 2, case["tokens"], host)
    if case["mixed"]:
        return before, torch.tensor([1] * (batch - 1) + [new])[torch.randperm(batch, generator=host)]
    return before, _spread(batch, max(1, new // 2 if new > 8 else 1), new, host) if case["ragged"] else torch.full((batch,), new)


def _prepare_chunk(case, gen, host):
    block, heads, dim, group = case["block"], case["heads"], case["dim"], case["group"]
    before, new = _chunk_lens(case, host)
    lens = before + new if case["causal"] else before.clamp(min=1)
    need = _up(lens, block)
    n_blocks, width = int(need.sum()) + 3, int(need.max()) + 2
    order = torch.randperm(n_blocks, generator=host).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    table[torch.arange(width)[None] < need[:, None]] = order[:int(need.sum())]
    K = _pool(gen, n_blocks, heads, block, dim, case["dtype"])
    V = torch.empty_like(K).normal_(generator=gen)
    deg = None
    if case["degrees"]:
        deg = _degrees(gen, K.shape[:3])
        if case["causal"]:                           # new tokens have degree 1
            for b in range(len(lens)):
                t = torch.arange(int(before[b]), int(lens[b]))
                deg[table[b, t // block].long().to(DEV), :, (t % block).to(DEV)] = 1
    n = int(new.sum()) + case["pad"]
    q = torch.empty((n, heads * group + 2 * heads, dim), device=DEV).normal_(generator=gen).to(K.dtype)   # a fused projection's output
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    return dict(kind="chunk", q=q[:, :heads * group], K=K, V=V, deg=deg, table=table.to(DEV), lens=_int(lens), starts=_int(starts),
                max_len=int(lens.max()), causal=case["causal"], host_lens=lens.tolist(), host_starts=starts.tolist(),
                out=torch.zeros((n, heads * group, dim), dtype=K.dtype, device=DEV),
                ws=torch.zeros(_SCRATCH, dtype=torch.uint8, device=DEV))


def _prepare_fork(case, gen, host):
    block, heads, dim, copies = case["block"], case["heads"], case["dim"], case["copies"]
    lens = _spread(case["sources"], max(case["tokens"] // 2, 1), case["tokens"], host)
    rows = case["sources"] * (1 + copies)
    own_rows = torch.arange(case["sources"]) * (1 + copies)      # a prompt's row, then those that continue it
    row_lens = torch.zeros(rows, dtype=torch.int64)
    row_lens[own_rows] = lens
    source = torch.full((rows,), -1)
    for i in range(1, copies + 1):
        source[own_rows + i] = own_rows
    need = _up(lens, block)
    used, asked = int(need.sum()), int(need.sum()) * copies
    spare = max(1, asked * 3 // 4) if case["short"] else asked + 5
    n_blocks, width = used + spare, int(need.max()) + 2
    order = torch.randperm(n_blocks, generator=host).to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32)
    mine = torch.full((case["sources"], width), -1, dtype=torch.int32)
    mine[torch.arange(width)[None] < need[:, None]] = order[:used]
    table[own_rows] = mine
    free = torch.full((4 + 2 * n_blocks,), -1, dtype=torch.int32)
    free[:4] = 0
    free[0] = spare
    free[4:4 + spare] = order[used:]
    free[4 + n_blocks:][order[:used].long()] = _IN_USE
    K = _pool(gen, n_blocks, heads, block, dim, case["dtype"])
    V = torch.empty_like(K).normal_(generator=gen)
    deg = _degrees(gen, K.shape[:3])
    bounds, mass = torch.stack([K.amin(2), K.amax(2)], 2), deg.sum(2, dtype=torch.int32)
    n_moves = asked + 1
    return dict(kind="fork", table=table.to(DEV), lens=_int(row_lens), before=_int(row_lens), source=_int(source), free=free.to(DEV),
                block=block, n_moves=n_moves, K=K, V=V, deg=deg, bounds=bounds, mass=mass,
                out=(_int(torch.zeros(n_moves, 2)), _int(torch.zeros(rows))))


def _compact_lens(case, host):
    """Lengths of the rows: of each pair the second is at least as long as the first."""
    v = np.linspace(max(case["tokens"] // 2, 1), case["tokens"], 2 * case["pairs"]).round().astype(np.int64)
    return torch.from_numpy(v).view(-1, 2)[torch.randperm(case["pairs"], generator=host)].flatten()


def _prepare_compact(case, gen, host):
    block, heads, dim = case["block"], case["heads"], case["dim"]
    lens = _compact_lens(case, host)
    rows, need = len(lens), _up(lens, block)
    first = torch.arange(rows) % 2 == 0                          # the half that finishes first sits in the lowest blocks
    n_first, used = int(need[first].sum()), int(need.sum())
    n_blocks, width = used + 7, int(need.max()) + 1
    order = torch.cat([torch.randperm(n_first, generator=host), n_first + torch.randperm(used - n_first, generator=host)]).to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32)
    for half, ids in ((first, order[:n_first]), (~first, order[n_first:])):
        part = torch.full((rows // 2, width), -1, dtype=torch.int32)
        part[torch.arange(width)[None] < need[half][:, None]] = ids
        table[half] = part
    free = torch.full((4 + 2 * n_blocks,), -1, dtype=torch.int32)
    free[:4] = 0
    free[0] = n_blocks - used
    free[4:4 + n_blocks - used] = torch.arange(n_blocks - 1, used - 1, -1)
    free[4 + n_blocks:4 + n_blocks + used] = _IN_USE
    K = _pool(gen, n_blocks, heads, block, dim, case["dtype"])
    V = torch.empty_like(K).normal_(generator=gen)
    halves = []
    for half in (first, ~first):
        new = torch.where(half, lens, 0)
        n_slots = int(new.sum())
        n_moves = int(need[half].sum()) + 1                      # (as many blocks as become free below the others')
        halves.append(dict(cut=_int(torch.where(half, 0, lens)), new=_int(new), n_slots=n_slots, n_moves=n_moves,
                           out=(_int(torch.zeros(n_moves, 2)), _int(torch.zeros(1))),
                           slots=tuple(_int(torch.zeros(n)) for n in (n_slots, rows + 1, rows))))
    return dict(kind="compact", table=table.to(DEV), lens=_int(lens), free=free.to(DEV), block=block, halves=halves, K=K, V=V,
                deg=_degrees(gen, K.shape[:3]), ws=torch.zeros(16 * n_blocks + (1 << 16), dtype=torch.uint8, device=DEV))


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if kind == "chunk":
        return _own_chunk(s) if own else _plain_chunk(s)
    if kind == "fork":
        return _own_fork(s) if own else _plain_fork(s)
    return _own_compact(s) if own else _plain_compact(s)


def _own_chunk(s):
    import paper_2506_11418_amd as ckv
    return ckv.paged_chunk_attn(s["q"], s["K"], s["V"], s["deg"], s["table"], s["lens"], s["starts"], s["max_len"], causal=s["causal"],
                                out=s["out"], workspace=s["ws"])


def _own_fork(s):
    import paper_2506_11418_amd as ckv
    moves, granted = ckv.paged_fork(s["table"], s["lens"], s["source"], s["free"], s["block"], s["n_moves"], out=s["out"])
    ckv.paged_copy(moves, s["K"], s["V"], s["deg"], s["bounds"], s["mass"])
    ckv.paged_trim(s["table"], s["lens"], s["before"], s["free"], s["block"])
    return moves, granted, s["table"], s["lens"], s["free"], s["K"], s["V"], s["deg"], s["bounds"], s["mass"]


def _own_compact(s):
    import paper_2506_11418_amd as ckv
    for half in s["halves"]:
        ckv.paged_trim(s["table"], s["lens"], half["cut"], s["free"], s["block"])
        moves, extent = ckv.paged_compact(s["table"], s["lens"], s["free"], s["block"], half["n_moves"], out=half["out"], workspace=s["ws"])
        ckv.paged_copy(moves, s["K"], s["V"], s["deg"])
        ckv.paged_reserve(s["table"], s["lens"], half["new"], s["free"], s["block"], half["n_slots"], out=half["slots"])
    return [h["out"][0] for h in s["halves"]] + [h["out"][1] for h in s["halves"]] + [s["table"], s["lens"], s["free"], s["K"], s["V"], s["deg"]]


def _scale(dim):
    return float(np.float32(1.0) / np.sqrt(np.float32(dim)))


def _plain_chunk(s):
    q, out, block = s["q"], s["out"], s["K"].shape[2]
    heads, dim = s["K"].shape[1], s["K"].shape[3]
    group, scale, starts = q.shape[1] // heads, _scale(dim), s["host_starts"]
    for b, n in enumerate(s["host_lens"]):
        lo, hi = starts[b], starts[b + 1]
        blk = s["table"][b, :_up(n, block)].long()
        k, v = (p[blk].transpose(0, 1).reshape(heads, -1, dim)[:, :n].float() for p in (s["K"], s["V"]))
        mine = q[lo:hi].float().view(hi - lo, heads, group, dim).permute(1, 0, 2, 3).reshape(heads, -1, dim)
        x = torch.matmul(mine, k.transpose(1, 2)).mul_(scale).view(heads, hi - lo, group, n)
        if s["deg"] is not None:
            x += torch.log(s["deg"][blk].transpose(0, 1).reshape(heads, -1)[:, :n].float())[:, None, None]
        if s["causal"]:
            at = torch.arange(n - (hi - lo), n, device=DEV)
            x.masked_fill_((torch.arange(n, device=DEV)[None] > at[:, None])[None, :, None], -math.inf)
        w = x.sub_(x.amax(3, keepdim=True)).exp_()
        total = w.sum(3, keepdim=True).view(heads, -1, 1)
        o = torch.matmul(w.view(heads, -1, n), v) / total
        out[lo:hi] = o.view(heads, hi - lo, group, dim).permute(1, 0, 2, 3).reshape(hi - lo, heads * group, dim).to(q.dtype)
    return out


def _plain_copy(moves, pools):
    """Pairs of -1 copy the first pair's source onto itself."""
    none = moves[:, 0] < 0
    src, dst = (torch.where(none, moves[0, 0].clamp(min=0), moves[:, i]).long() for i in (0, 1))
    for p in pools:
        p[dst] = p[src]


def _plain_fork(s):
    table, lens, free, block, n_moves = s["table"], s["lens"], s["free"], s["block"], s["n_moves"]
    n_blocks, (rows, width) = (len(free) - 4) // 2, table.shape
    stack, marks, count = free[4:4 + n_blocks], free[4 + n_blocks:], free[0].long()
    L, src = lens.long(), s["source"].long()
    row = torch.arange(rows, device=DEV)
    asked = (src >= 0) & (src < rows) & (src != row) & (L == 0)
    length = torch.where(asked, L[src.clamp(0, rows - 1)], 0)
    need = (length + block - 1) // block
    ends = need.cumsum(0)
    granted = asked & ((need == 0) | ((ends <= count) & (ends <= n_moves)))
    take = torch.where(granted, need, 0)
    base = take.cumsum(0) - take
    k = torch.arange(width, device=DEV)[None]
    fresh = k < take[:, None]
    place = base[:, None] + k
    old = table[src.clamp(0, rows - 1)]
    dealt = stack[(count - 1 - place).clamp(0, n_blocks - 1)]
    moves = s["out"][0].fill_(-1)
    slot = torch.where(fresh, place, n_moves).flatten()
    pairs = torch.cat([moves, moves[:1]])
    pairs.scatter_(0, slot[:, None].expand(-1, 2), torch.stack([old, dealt], 2).view(-1, 2))
    moves.copy_(pairs[:n_moves])
    table.copy_(torch.where(fresh, dealt, table))
    _plain_copy(moves, [s["K"], s["V"], s["deg"], s["bounds"], s["mass"]])
    s["out"][1].copy_(granted)
    # the rows that were forked give their blocks back: the stack and the marks are what they were
    table.copy_(torch.where(fresh, -1, table))
    return moves, s["out"][1], table, lens, free, s["K"], s["V"], s["deg"], s["bounds"], s["mass"]


def _plain_compact(s):
    table, lens, free, block = s["table"], s["lens"], s["free"], s["block"]
    n_blocks, (rows, width) = (len(free) - 4) // 2, table.shape
    stack, marks = free[4:4 + n_blocks], free[4 + n_blocks:]
    col, at = torch.arange(width, device=DEV)[None], torch.arange(n_blocks, device=DEV)
    for half in s["halves"]:
        # finished rows give their blocks back
        gone = (lens > half["cut"])[:, None] & (table >= 0)
        spot = torch.where(gone, table, n_blocks).flatten().long()
        freed = torch.zeros(n_blocks + 1, dtype=torch.bool, device=DEV).scatter_(0, spot, True)[:n_blocks]
        table.masked_fill_(gone, -1)
        lens.copy_(torch.minimum(lens, half["cut"]))
        # the highest blocks that are left move into the lowest free ones
        empty = freed | (marks == -1)
        inside = (col < _up(lens[:, None].long(), block)) & (table >= 0)
        spot = torch.where(inside, table, n_blocks).flatten().long()
        used = torch.zeros(n_blocks + 1, dtype=torch.bool, device=DEV).scatter_(0, spot, True)[:n_blocks]
        below = empty.long().cumsum(0)                           # free ones up to here
        above = used.long().flip(0).cumsum(0).flip(0)            # used ones from here on
        k = torch.minimum(below - empty.long(), above).amax().clamp(max=half["n_moves"])
        mover, home = used & (above <= k), empty & (below <= k)
        n_moves = half["n_moves"]
        pairs = torch.full((n_moves + 1, 2), -1, dtype=torch.int32, device=DEV)
        number = at.to(torch.int32)
        pairs[:, 0].scatter_(0, torch.where(mover, k - above, n_moves), number)
        pairs[:, 1].scatter_(0, torch.where(home, below - 1, n_moves), number)
        moves, extent = half["out"]
        moves.copy_(pairs[:n_moves])
        _plain_copy(moves, [s["K"], s["V"], s["deg"]])
        renamed = torch.where(mover, pairs[(k - above).clamp(0, n_moves), 1], number)
        table.copy_(torch.where(inside, renamed[table.clamp(min=0).long()], table))
        empty = (empty & ~home) | mover
        marks.copy_(torch.where(empty, -1, _IN_USE))
        extent.copy_(torch.where(empty, 0, at + 1).amax()[None])
        left = empty.sum()
        place = torch.where(empty, left - empty.long().cumsum(0), n_blocks)
        full = torch.full((n_blocks + 1,), -1, dtype=torch.int32, device=DEV).scatter_(0, place, number)
        stack.copy_(full[:n_blocks])
        # new rows
        need = _up(half["new"].long(), block)
        base = need.cumsum(0) - need
        fresh = col < need[:, None]
        table.copy_(torch.where(fresh, stack[(left - 1 - base[:, None] - col).clamp(0, n_blocks - 1)], table))
        taken = (at < left) & (at >= left - need.sum())
        spot = torch.where(taken, stack.long(), n_blocks)
        dealt = torch.zeros(n_blocks + 1, dtype=torch.bool, device=DEV).scatter_(0, spot, True)[:n_blocks]
        marks.masked_fill_(dealt, _IN_USE)
        lens.copy_(lens + half["new"])
        free[0] = left - need.sum()
    return [h["out"][0] for h in s["halves"]] + [h["out"][1] for h in s["halves"]] + [table, lens, free, s["K"], s["V"], s["deg"]]


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    block, row = case["block"], case["heads"] * case["dim"] * (4 if case["dtype"] == "f32" else 2)
    if case["kind"] == "chunk":
        before, new = _chunk_lens(case, torch.Generator().manual_seed(1))    # (which row is how long: the seed's; their sums are not)
        lens = before + new if case["causal"] else before.clamp(min=1)
        seen = float((new * (lens - new) + new * (new + 1) // 2 if case["causal"] else new * lens).sum())
        cache, n = int(lens.sum()), int(new.sum())
        per_token = 2 * row + (4 * case["heads"] if case["degrees"] else 0)
        return dict(bytes=cache * per_token + 2 * n * case["group"] * row + 4 * int(_up(lens, block).sum()),
                    flops=4 * case["heads"] * case["group"] * case["dim"] * seen)
    page = block * (2 * row + 4 * case["heads"])
    host = torch.Generator().manual_seed(1)
    if case["kind"] == "fork":
        need = _up(_spread(case["sources"], max(case["tokens"] // 2, 1), case["tokens"], host), block)
        copied = float(need.sum()) * case["copies"] * (0.75 if case["short"] else 1)
        page += 2 * row + 4 * case["heads"]                                  # its bounds and its mass
        # a prompt's pages are read once however often they are written; pairs, entries, stack and mark of a block, there and back
        read = float(need.sum())
        return dict(bytes=page * (read + copied) + 32 * copied + 24 * case["sources"] * (1 + case["copies"]), flops=0)
    need = _up(_compact_lens(case, host), block)
    moved = 2 * float(need[::2].sum())                                       # each half fills what the shorter one has left
    return dict(bytes=moved * 2 * page + 40 * float(need.sum()) + 48 * len(need), flops=0)


# ---- the definitions in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"chunk": _exact_chunk, "fork": _exact_fork, "compact": _exact_compact}[s["kind"]](s)


def _exact_chunk(s):
    heads, block, dim = s["K"].shape[1:]
    q, o = s["q"].double(), s["out"].double()
    group, scale = q.shape[1] // heads, _scale(dim)
    for b, n in enumerate(s["host_lens"]):
        first, last = s["host_starts"][b:b + 2]
        ids = s["table"][b, :_up(n, block)].long()
        for h in range(heads):
            k, v = (p[ids, h].double().reshape(-1, dim)[:n] for p in (s["K"], s["V"]))
            extra = 0.0 if s["deg"] is None else s["deg"][ids, h].flatten()[:n].double().log()
            for lo in range(first, last, 4096):
                hi = min(lo + 4096, last)
                seen = n - (last - first) + hi - first if s["causal"] else n       # (the last of these tokens sees this many)
                kt = k[:seen].T.contiguous()
                for g in range(h * group, (h + 1) * group):
                    x = q[lo:hi, g] @ kt * scale
                    x = x + (extra if s["deg"] is None else extra[:seen])
                    if s["causal"]:
                        x = torch.where(torch.ones_like(x, dtype=torch.bool).tril(seen - (hi - lo)), x, -math.inf)
                    o[lo:hi, g] = torch.softmax(x, 1) @ v[:seen]
    return o


def _exact_fork(s):
    """The pages after the call, a row of the table after the other."""
    table, lens, source, block = s["table"].cpu(), s["lens"].tolist(), s["source"].tolist(), s["block"]
    count, stack = int(s["free"][0]), s["free"][4:].tolist()
    src, dst, asked = [], [], 0
    for b, f in enumerate(source):
        if f < 0:
            continue
        n = _up(lens[f], block)
        asked += n
        if n and asked <= min(count, s["n_moves"]):
            for i in range(n):
                src.append(int(table[f, i]))
                dst.append(stack[count - 1 - len(dst)])
    src, dst = torch.tensor(src, dtype=torch.int64, device=DEV), torch.tensor(dst, dtype=torch.int64, device=DEV)
    pages = []
    for p in (s["K"], s["V"], s["bounds"]):
        want = p.double()
        want.index_copy_(0, dst, want.index_select(0, src))
        pages.append(want)
    return None, None, None, None, None, pages[0], pages[1], None, pages[2], None


def _exact_compact(s):
    table, lens, block, n_blocks = s["table"].tolist(), s["lens"].tolist(), s["block"], s["K"].shape[0]
    K, V = s["K"].double(), s["V"].double()
    rows = {b: row[:_up(lens[b], block)] for b, row in enumerate(table)}
    for i in range(2):
        kept = {b: r for b, r in rows.items() if b % 2 != i}
        inside = set(x for r in kept.values() for x in r)
        free = [x for x in range(n_blocks) if x not in inside]
        high = sorted(inside, reverse=True)
        k = 0
        while k < min(len(free), len(high), s["halves"][i]["n_moves"]) and high[k] > free[k]:
            k += 1
        went = dict(zip(sorted(high[:k]), free[:k]))
        src, dst = (torch.tensor(list(x), dtype=torch.int64, device=DEV) for x in (went.keys(), went.values()))
        for p in (K, V):
            p.index_copy_(0, dst, p.index_select(0, src))
        rows = {b: [went.get(x, x) for x in r] for b, r in kept.items()}
        inside = set(x for r in rows.values() for x in r)
        fresh = iter(x for x in range(n_blocks) if x not in inside)
        for b in range(i, len(lens), 2):
            rows[b] = [next(fresh) for _ in range(_up(lens[b], block))]
    return [None] * 7 + [K, V, None]
