"""Block tables, slot maps and block selection of a paged cache, from their definitions, one request after the other.

The free list is a plain list of block numbers, dealt from its end, and a set of the blocks that are dealt.
"""
from __future__ import annotations

import math

import numpy as np


class FreeList:
    def __init__(self, n_blocks: int, free=None):
        """free: the free blocks, the last one dealt first (default: all, block 0 first)."""
        self.n_blocks = n_blocks
        self.stack = list(range(n_blocks - 1, -1, -1)) if free is None else [int(x) for x in free]
        self.dealt = set(range(n_blocks)) - set(self.stack)

    def back(self, ids) -> None:
        """The blocks of `ids` that are dealt return, the last first; each once."""
        for blk in [int(x) for x in ids][::-1]:
            if blk in self.dealt:
                self.dealt.remove(blk)
                self.stack.append(blk)


def reserve(table, lens, n_new, free: FreeList, block: int, n_slots: int):
    """Updates table [batch, width], lens and free; returns (slots, starts, granted) as lists."""
    batch, width = table.shape
    slots, starts, granted = [], [0], []
    tokens = asked = 0
    n_free = len(free.stack)
    for b in range(batch):
        L, n = int(lens[b]), max(int(n_new[b]), 0)
        tokens += n
        fits = L >= 0 and L + n <= width * block and tokens <= n_slots
        need = -(-(L + n) // block) - (-(-L // block)) if fits else 0
        asked += need
        ok = fits and (need == 0 or asked <= n_free)
        granted.append(int(ok))
        if ok:
            first = -(-L // block)
            for k in range(need):
                table[b, first + k] = free.stack.pop()
                free.dealt.add(int(table[b, first + k]))
            lens[b] = L + n
        for t in range(L, L + min(n, max(n_slots - len(slots), 0))):
            blk = int(table[b, t // block]) if ok else -1
            slots.append(blk * block + t % block if 0 <= blk < free.n_blocks else -1)
        starts.append(min(tokens, n_slots))
    return slots + [-1] * (n_slots - len(slots)), starts, granted


def trim(table, lens, new_lens, free: FreeList, block: int) -> None:
    gone = []
    for b in range(table.shape[0]):
        L, cut = int(lens[b]), int(new_lens[b])
        if 0 <= cut < L:
            last = min(-(-L // block), table.shape[1])
            gone += table[b, -(-cut // block):last].tolist()
            table[b, -(-cut // block):last] = -1
            lens[b] = cut
    free.back(gone)


def bounds(K, deg):
    """K [tokens, dim], deg [tokens] of one (block, head): (lo, hi, mass) over the tokens of degree 1 and more."""
    keep = np.asarray(deg) > 0
    k = np.asarray(K, dtype=np.float64)[keep]
    if not keep.any():
        return np.full(K.shape[1], np.inf), np.full(K.shape[1], -np.inf), 0
    return k.min(0), k.max(0), int(np.asarray(deg)[keep].sum())


def scores(q, lo, hi, mass, scale):
    """q [group, dim] of one KV head against blocks lo, hi [n, dim], mass [n]: the upper bounds of ln(sum of deg * exp(scale q.k)),
    summed in extended precision and rounded once, fp32."""
    q, lo, hi = (np.asarray(x, dtype=np.longdouble) for x in (q, lo, hi))
    with np.errstate(all="ignore"):
        dots = np.stack([np.maximum(x * lo, x * hi).sum(1) for x in q])
        s = dots.max(0) * np.longdouble(scale) + np.log(np.asarray(mass, dtype=np.longdouble))
        odd = ~np.isfinite(lo).all(1) | ~np.isfinite(hi).all(1) | (not np.isfinite(q).all())
    return np.where(odd, np.nan, s).astype(np.float32)


def select(scores, n: int, n_select: int, n_sink: int, n_recent: int):
    """Positions, ascending, of the blocks to read; scores[i] is a number (one that is not
    finite comes before those that are) or "out" for a block without mass or outside the pool."""
    def rank(i):
        s = scores[i]
        if i < n_sink or i >= n - n_recent:
            return (0, 0.0, i)
        if s == "out":
            return (3, 0.0, i)
        if not math.isfinite(s):
            return (1, 0.0, i)
        return (2, -s, i)
    return sorted(sorted(range(n), key=rank)[:n_select])
