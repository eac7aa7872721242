"""The paged oracle against its own definitions, without a GPU."""
import math

import numpy as np
import pytest

from oracle import paged_oracle as po


def test_a_reservation_taken_back_leaves_everything_as_it_was():
    rng = np.random.default_rng(1)
    for _ in range(50):
        batch, width, block = int(rng.integers(1, 6)), int(rng.integers(1, 9)), int(rng.choice([1, 4, 16]))
        free = po.FreeList(batch * width + 3)
        table, lens = np.full((batch, width), -1), np.zeros(batch, dtype=np.int64)
        po.reserve(table, lens, rng.integers(0, width * block + 1, batch), free, block, 10**6)
        t0, l0, s0 = table.copy(), lens.copy(), list(free.stack)
        _, _, ok = po.reserve(table, lens, rng.integers(0, block * 2, batch), free, block, 10**6)
        po.trim(table, lens, l0, free, block)
        assert np.array_equal(table, t0) and np.array_equal(lens, l0) and free.stack == s0


def test_slots_of_a_small_step():
    free = po.FreeList(4, [3, 1, 0, 2])
    table, lens = np.full((2, 3), -1), np.array([0, 0])
    slots, starts, ok = po.reserve(table, lens, [3, 2], free, 2, 6)
    assert table.tolist() == [[2, 0, -1], [1, -1, -1]] and slots == [4, 5, 0, 2, 3, -1] and starts == [0, 3, 5] and ok == [1, 1]
    slots, starts, ok = po.reserve(table, lens, [4, 1], free, 2, 6)      # a row of three blocks; one block left
    assert ok == [0, 1] and slots == [-1] * 4 + [6] + [-1] and lens.tolist() == [3, 3]


@pytest.mark.parametrize("seed", range(4))
def test_the_score_bounds_the_softmax_mass_of_its_block(seed):
    rng = np.random.default_rng(seed)
    for _ in range(20):
        K, deg, q = rng.normal(size=(16, 32)), rng.integers(0, 5, 16), rng.normal(size=(4, 32))
        deg[0] = 1
        lo, hi, mass = po.bounds(K, deg)
        keep = deg > 0
        true = max(math.log((deg[keep] * np.exp(0.2 * K[keep] @ x)).sum()) for x in q)
        assert po.scores(q, lo[None], hi[None], [mass], 0.2)[0] >= true - 1e-5


def test_selection_order():
    s = [0.0, 5.0, math.nan, "out", 5.0, 7.0, 1.0, 2.0]
    assert po.select(s, 8, 2, 1, 1) == [0, 7]
    assert po.select(s, 8, 4, 1, 1) == [0, 2, 5, 7]
    assert po.select(s, 8, 5, 1, 1) == [0, 1, 2, 5, 7]
    assert po.select(s, 8, 7, 1, 1) == [0, 1, 2, 4, 5, 6, 7]
