"""The native binding makes the calls for new tokens over pages itself, with arguments in the library's order, and gives the bits of the ctypes
route; and calls on two streams at once, each with buffers of its own."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_chunk import _close, _oracle, _queries, _starts
from test_gpu_sparse import DEV, Cache, _dev, _scale
from test_gpu_write_strides import _Never, _Recorder

pytestmark = pytest.mark.gpu


def _pool(c):
    """A cache on the GPU with the free list that goes with its table."""
    K, V, deg, table, lens = c.gpu()
    free, used = ckv.paged_free_list(c.n_blocks), sorted(set(table[table >= 0].tolist()))
    left = [x for x in range(c.n_blocks) if x not in used]
    free[0] = len(left)
    free[4:4 + len(left)] = _dev(left)
    free[4 + c.n_blocks:][torch.tensor(used, device=DEV)] = 2**31 - 1
    return K, V, deg, table, lens, free


@pytest.mark.parametrize("dtype,degrees,bounds", [("bf16", True, True), ("f32", False, False)])
def test_the_binding_makes_every_call(monkeypatch, dtype, degrees, bounds):
    block, heads, dim = 16, 2, 64
    native, outs = _Recorder(ckv._binding()), []
    for module in (native, _Never()):
        monkeypatch.setattr(ckv, "_native", module)
        c = Cache(23, [200, 0, 77], heads, dim, block, dtype, degrees, spare=30)
        K, V, deg, table, lens, free = _pool(c)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        b = (torch.ones(c.n_blocks, heads, 2, dim, dtype=c.dtype, device=DEV), i32(c.n_blocks, heads)) if bounds else (None, None)
        moves, granted = ckv.paged_fork(table, lens, _dev([-1, 0, -1]), free, block, 15, out=(i32(15, 2), i32(3)))
        ckv.paged_copy(moves, K, V, deg, *b)
        q = _queries(3, 30, heads * 4, dim, c.dtype).to(DEV)
        ws = torch.zeros(ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), heads * 4, 30, 200), dtype=torch.uint8, device=DEV)
        o = ckv.paged_chunk_attn(q, K, V, deg, table, lens, _dev([0, 10, 20, 30]), 200, scale=0.25, causal=False,
                                 out=torch.zeros(q.shape, device=DEV), workspace=ws)
        ckv.paged_trim(table, lens, _dev([0, -1, -1]), free, block)
        ws = torch.zeros(ckv.paged_compact_workspace(c.n_blocks), dtype=torch.uint8, device=DEV)
        down, extent = ckv.paged_compact(table, lens, free, block, 40, out=(i32(40, 2), i32(1)), workspace=ws)
        ckv.paged_copy(down, K, V, deg, *b)
        torch.cuda.synchronize()
        assert torch.equal(o[:10], ckv.paged_chunk_attn(q[:10], K, V, deg, table[1:2].contiguous(), lens[1:2].clone(), _dev([0, 10]), 200, scale=0.25,
                                                        causal=False, out_dtype=torch.float32))       # the copy answers as its source did
        outs.append([K, V, table, lens, free, moves, granted, o, down, extent] + [x for x in (deg, *b) if x is not None])
    names = ["paged_fork", "paged_copy", "paged_chunk_attn", "paged_trim", "paged_compact", "paged_copy"]
    assert native.took[:len(names)] == [(n, 0) for n in names]
    for x, y in zip(*outs):
        assert torch.equal(x.nan_to_num(), y.nan_to_num()) if x.is_floating_point() else torch.equal(x, y)
    assert outs[0][6].tolist() == [0, 1, 0]


def test_two_streams_at_once():
    """Attention over one cache while another pool is forked, copied and compacted: each stream with its own buffers."""
    lens, new = [900, 300], [100, 60]
    c = Cache(29, lens, 2, 128, 16)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new)
    q = _queries(4, starts[-1], 8, 128, c.dtype)
    want, bound = _oracle(c, q, new, starts, True, _scale(128))
    other = Cache(37, [500, 0, 0], 4, 64, 8, spare=200)
    fresh = [x.clone() for x in _pool(other)]
    state = [x.clone() for x in fresh]
    streams, dev = [torch.cuda.Stream() for _ in range(2)], q.to(DEV)
    torch.cuda.synchronize()
    outs, pairs = [], []
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            outs.append(ckv.paged_chunk_attn(dev, K, V, deg, table, n, _dev(starts), 900))
        with torch.cuda.stream(streams[1]):
            pk, pv, pd, pt, pl, pf = state
            for x, y in zip((pt, pl, pf), fresh[3:]):
                x.copy_(y)
            moves, granted = ckv.paged_fork(pt, pl, _dev([-1, 0, 0]), pf, 8, 126)
            ckv.paged_copy(moves, pk, pv, pd)
            pairs.append((moves, granted, pt.clone(), pl.clone()))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, outs[0])
    _close(outs[0], want, bound, c.dtype)
    for p in pairs:
        assert all(torch.equal(x, y) for x, y in zip(p, pairs[0])) and p[1].tolist() == [0, 1, 1] and p[3].tolist() == [500] * 3
    row = [state[0][state[3][b, :63].long()] for b in range(3)]
    assert all(torch.equal(x.nan_to_num(), row[0].nan_to_num()) for x in row)


def test_lengths_below_the_new_tokens_and_tables_of_one_block():
    """One page for everything: the longest sequence a table holds, and tokens before the first."""
    c = Cache(43, [16, 3], 1, 64, 16, room=0)
    K, V, deg, table, n = c.gpu()
    assert table.shape == (2, 1)
    q = _queries(5, 24, 8, 64, c.dtype)
    want, bound = _oracle(c, q, [16, 8], [0, 16, 24], True, _scale(64))
    got = ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev([0, 16, 24]), 1 << 20)
    _close(got, want, bound, c.dtype)
    assert (got[16:21] == 0).all() and np.abs(want[21:]).min() > 0
