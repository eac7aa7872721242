"""Two calls for new tokens and a pool's forks, trims, compactions and copies on three streams at once, each with buffers of its own."""
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_chunk import _close, _oracle, _queries, _starts
from test_gpu_chunk_parts import _is_cut
from test_gpu_pages_routes import _pool
from test_gpu_sparse import DEV, Cache, _dev, _scale

pytestmark = pytest.mark.gpu


class _Attention:
    """A call that is cut, with a workspace of its own."""

    def __init__(self, seed, lens, new, causal):
        self.c, self.causal = Cache(seed, lens, 2, 128, 16), causal
        self.starts, self.new = _starts(new), new
        self.q = _queries(seed, self.starts[-1], 8, 128, self.c.dtype)
        K, V, deg, table, n = self.c.gpu()
        self.args = (self.q.to(DEV), K, V, deg, table, n, _dev(self.starts), max(lens))
        assert _is_cut(*self.args, causal=causal)
        self.ws = torch.full((ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), 8, self.q.shape[0], max(lens)),), 255, dtype=torch.uint8, device=DEV)

    def __call__(self):
        return ckv.paged_chunk_attn(*self.args, causal=self.causal, out=torch.zeros_like(self.args[0]), workspace=self.ws)

    def check(self, got):
        want, bound = _oracle(self.c, self.q, self.new, self.starts, self.causal, _scale(128))
        _close(got, want, bound, self.c.dtype)


class _Pool:
    """Rows forked, the ones they continue dropped, the pool compacted; the whole from the same state every time."""

    def __init__(self, seed, lens, block, spare):
        self.c = Cache(seed, lens, 1, 64, block, spare=spare)
        self.fresh = [x.clone() for x in _pool(self.c)]
        self.K, self.V, self.deg, self.table, self.lens, self.free = (x.clone() for x in self.fresh)
        self.source = _dev([b - 1 if n == 0 else -1 for b, n in enumerate(lens)])
        self.kept = _dev([0] * len(lens))
        for b, n in enumerate(lens):
            if n == 0:
                self.kept[b] = lens[b - 1]
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        self.used = sum(-(-n // block) for n in lens)
        self.moves, self.granted, self.down, self.extent = i32(self.used, 2), i32(len(lens)), i32(self.used, 2), i32(1)
        self.ws = torch.full((ckv.paged_compact_workspace(self.c.n_blocks),), 255, dtype=torch.uint8, device=DEV)

    def __call__(self):
        for x, y in zip((self.K, self.V, self.deg, self.table, self.lens, self.free), self.fresh):
            x.copy_(y)
        block = self.c.block
        ckv.paged_fork(self.table, self.lens, self.source, self.free, block, self.used, out=(self.moves, self.granted))
        ckv.paged_copy(self.moves, self.K, self.V, self.deg)
        ckv.paged_trim(self.table, self.lens, self.kept, self.free, block)
        ckv.paged_compact(self.table, self.lens, self.free, block, self.used, out=(self.down, self.extent), workspace=self.ws)
        ckv.paged_copy(self.down, self.K, self.V, self.deg)
        return [x.clone() for x in (self.table, self.lens, self.free, self.moves, self.granted, self.down, self.extent, self.K, self.V, self.deg)]

    def check(self, got):
        table, lens, free, _, granted, down, extent, K, V, deg = got
        assert int(extent) == self.used and int(free[0]) == self.c.n_blocks - self.used and int((down[:, 0] >= 0).sum()) > 0
        old_table = self.fresh[3]
        for b, n in enumerate(self.c.lens):
            if n:
                assert int(lens[b]) == 0 and int(granted[b]) == 0
                continue
            m = self.c.lens[b - 1]
            assert int(lens[b]) == m and int(granted[b]) == 1
            at, was = table[b, :-(-m // self.c.block)].long(), old_table[b - 1, :-(-m // self.c.block)].long()
            for pool, old in zip((K, V, deg), self.fresh):
                assert torch.equal(pool[at].nan_to_num(), old[was].nan_to_num())


@pytest.mark.parametrize("lens,block,spare", [([16001, 0, 9000, 0], 4, 6300), ([700, 0, 333, 0], 8, 140)])
def test_three_streams_at_once(lens, block, spare):
    """(The first pool has more entries than one workgroup settles, so that the steps through the workspace run; the second has not.)"""
    print(f"streams {lens} block {block}", flush=True)
    calls = [_Attention(29, [900, 300], [100, 60], True), _Attention(31, [700, 1100, 40], [30, 9, 2], False), _Pool(37, lens, block, spare)]
    assert (len(lens) * calls[2].table.shape[1] > 8192) == (block == 4)
    alone = [f() for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = [[] for _ in calls]
    for _ in range(5):
        for f, s, o in zip(calls, streams, outs):
            with torch.cuda.stream(s):
                o.append(f())
    torch.cuda.synchronize()
    for f, first, many in zip(calls, alone, outs):
        f.check(first)
        for o in many:
            pairs = [(first, o)] if torch.is_tensor(o) else zip(first, o)
            assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) if x.is_floating_point() else torch.equal(x, y) for x, y in pairs)
