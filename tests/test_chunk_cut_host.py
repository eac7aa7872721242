"""How many parts a call for new tokens is cut into, seen in the workspace that it needs.  No GPU needed."""
import ctypes as C

import numpy as np
import pytest

import paper_2506_11418_amd as ckv

EWORKSPACE, EINVAL = -4, -1


def _p(i):
    return C.c_void_p(i << 42)                   # far apart, never followed


def _need(batch, n, max_len, heads=8, q_heads=32, dim=128):
    """The least workspace that a call takes.  Its output lies over its queries, which is found after the workspace is large enough."""
    pl = ckv.PagedLayout(batch, heads, dim, ckv.BF16, 16, -(-max_len // 16), 1000)

    def refused(size):
        st = ckv.lib().ckv_paged_chunk_attn(_p(1), q_heads * dim, dim, q_heads, _p(2), n, _p(3), _p(4), None, _p(6), _p(7), C.byref(pl), max_len, 0.0, 1,
                                            _p(1), ckv.BF16, _p(9), size, None)
        assert st in (EWORKSPACE, EINVAL)
        return st == EWORKSPACE
    lo, hi = -1, 1 << 32
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if refused(mid) else (lo, mid)
    return hi


@pytest.mark.parametrize("n,max_len", [(1, 32768), (3, 32768), (8, 5000), (33, 16384), (40, 1000)])
def test_rows_of_the_table_without_new_tokens_change_nothing(n, max_len):
    """A table has as many rows as a server has places for requests; n tokens belong to n of them at most."""
    need = _need(max(n, 2), n, max_len)
    assert need > 0
    for batch in (64, 65, 192, 256, 1000, 4096, 65535):
        assert _need(batch, n, max_len) == need, batch


def test_workspace_of_more_rows_than_new_tokens():
    """What the query for a size names is enough for any batch."""
    for n in (1, 7, 64, 65, 100, 500):
        for max_len in (100, 1000, 16384, 1 << 20):
            for heads, q_heads in ((8, 32), (1, 8), (2, 2), (40, 40)):
                for batch in (1, 64, 65, 300, 65535):
                    pl = ckv.PagedLayout(batch, heads, 128, ckv.BF16, 16, -(-max_len // 16), 1000)
                    assert _need(batch, n, max_len, heads, q_heads) <= ckv.paged_chunk_attn_workspace(pl, q_heads, n, max_len), (n, max_len, heads, batch)


@pytest.mark.parametrize("seed", range(40))
def test_places_of_many_sequences(seed):
    """The rule by which a workgroup finds its tokens in a batch of more than 64: sequence b's places begin at starts[b] // T + min(starts[b], b).  Every
    token has one place, among n // T + min(n, batch) of them."""
    rng = np.random.default_rng(seed)
    for T in (16, 32, 64, 128):
        batch = int(rng.integers(65, 400))
        new = rng.integers(0, int(rng.choice([2, 3, 40, 300])), batch) * (rng.random(batch) < rng.choice([0.02, 0.5, 1.0]))
        starts = int(rng.choice([0, 5, 77])) + np.concatenate([[0], np.cumsum(new)])
        n = int(starts[-1]) + int(rng.choice([0, 9]))
        first = starts[:-1] // T + np.minimum(starts[:-1], np.arange(batch))
        seen = []
        for place in range(n // T + min(max(n, 1), batch)):
            b = int((first <= place).sum()) - 1
            if b >= 0:
                at = int(starts[b]) + (place - int(first[b])) * T
                seen += range(at, min(at + T, int(starts[b + 1])))
        assert seen == list(range(int(starts[0]), int(starts[-1])))
