"""The oracle of new tokens' attention, forks and compactions against their definitions, without a GPU."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po


def _tables(rng):
    batch, width, block = int(rng.integers(2, 7)), int(rng.integers(1, 8)), int(rng.choice([1, 4, 16]))
    free = po.FreeList(batch * width + int(rng.integers(0, 9)))
    table, lens = np.full((batch, width), -1), np.zeros(batch, dtype=np.int64)
    po.reserve(table, lens, rng.integers(0, width * block + 1, batch), free, block, 10**6)
    return table, lens, free, block


def _rows(table, lens, block):
    return [[int(x) for x in table[b, :-(-int(n) // block)]] for b, n in enumerate(lens)]


@pytest.mark.parametrize("seed", range(6))
def test_attention_is_the_weighted_mean(seed):
    """Each token counted deg times, one after the other, with exponentials of differences."""
    rng = np.random.default_rng(seed)
    n, heads, tokens, dim = 3, 2, int(rng.integers(1, 9)), 4
    q, k, v = rng.normal(size=(n, heads, dim)), rng.normal(size=(tokens, dim)), rng.normal(size=(tokens, dim))
    deg, seen = rng.integers(-1, 4, tokens), rng.integers(-2, tokens + 1, n)
    o, a, x = po.chunk_attention(q, k, v, deg, seen, 0.3)
    for i in range(n):
        for h in range(heads):
            num, den, most = np.zeros(dim), 0.0, 0.0
            for t in range(max(int(seen[i]), 0)):
                for _ in range(max(int(deg[t]), 0)):
                    w = math.exp(0.3 * float(q[i, h] @ k[t]))
                    num, den = num + w * v[t], den + w
                    most = max(most, float(np.abs(q[i, h] * k[t]).sum()))
            assert np.allclose(o[i, h], num / den if den else 0.0, rtol=1e-12, atol=1e-14) and abs(x[i, h] - most) < 1e-12
            assert (a[i, h] >= np.abs(o[i, h]) - 1e-14).all()


def test_attention_where_nothing_or_no_number_is_seen():
    q, k, v, one = np.ones((1, 1, 2)), np.array([[1.0, 0.0], [np.inf, 0.0]]), np.ones((2, 2)), np.array([1, 1])
    assert (po.chunk_attention(q, k, v, one, [0], 1.0)[0] == 0).all()
    assert (po.chunk_attention(q, k, v, one, [1], 1.0)[0] == 1).all()
    assert np.isnan(po.chunk_attention(q, k, v, one, [2], 1.0)[0]).all()
    assert (po.chunk_attention(q, k, v, np.array([1, 0]), [2], 1.0)[0] == 1).all()
    assert (po.chunk_attention(-q, k, v, one, [2], 1.0)[0] == 1).all()         # a logit of -inf has no weight


@pytest.mark.parametrize("seed", range(20))
def test_forked_rows_hold_copies_and_are_taken_back_by_a_trim(seed):
    rng = np.random.default_rng(seed)
    table, lens, free, block = _tables(rng)
    lens[0], gone = 0, _rows(table, lens, block)[0]
    free.back([int(x) for x in table[0] if x >= 0])
    table[0] = -1
    t0, l0, s0 = table.copy(), lens.copy(), list(free.stack)
    source = np.full(len(lens), -1)
    source[0] = f = int(rng.integers(1, len(lens)))
    moves, granted = po.fork(table, lens, source, free, block, 10**6)
    need = len(_rows(t0, l0, block)[f])
    if need > len(s0):
        assert not any(granted) and not moves and np.array_equal(table, t0)
        return
    assert granted[0] == 1 and sum(granted) == 1 and lens[0] == l0[f]
    rows = _rows(table, lens, block)
    assert moves == list(zip(rows[f], rows[0])) and not set(rows[0]) & set(rows[f]) and len(set(rows[0])) == need
    assert len(set(sum(rows, []))) == len(sum(rows, []))                        # a block belongs to one row
    po.trim(table, lens, l0, free, block)
    assert np.array_equal(table, t0) and np.array_equal(lens, l0) and free.stack == s0


@pytest.mark.parametrize("seed", range(20))
def test_compacted_blocks_hold_what_they_held(seed):
    rng = np.random.default_rng(seed)
    table, lens, free, block = _tables(rng)
    keep = rng.random(len(lens)) < 0.5
    po.trim(table, lens, np.where(keep, lens, 0), free, block)
    held = {x: f"page {x}" for x in free.dealt}
    before = [[held[x] for x in r] for r in _rows(table, lens, block)]
    n_dealt, most = len(free.dealt), int(rng.choice([0, 1, 2, 99]))
    moves, extent = po.compact(table, lens, free, block, most)
    assert len(moves) <= most and all(to < at for at, to in moves) and not {x for x, _ in moves} & {y for _, y in moves}
    for at, to in moves:
        held[to] = held[at]
    assert [[held[x] for x in r] for r in _rows(table, lens, block)] == before
    assert len(free.dealt) == n_dealt and set(sum(_rows(table, lens, block), [])) == free.dealt
    assert extent == max(free.dealt, default=-1) + 1 and (most < 99 or extent == n_dealt)
    assert free.stack == sorted(set(range(free.n_blocks)) - free.dealt, reverse=True)
    if most == 99:
        assert po.compact(table, lens, free, block, 99) == ([], extent)       # twice is once
