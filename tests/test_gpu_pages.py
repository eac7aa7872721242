"""Rows forked, pages compacted and copied on the GPU, against the oracle's one request after the other: whole numbers and copies, so
everything has to be equal; and a run of the paged calls together, as a serving program makes them."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from oracle import paged_oracle as po
from parity_util import f64
from test_gpu_chunk import _close, _oracle, _queries, _starts
from test_gpu_sparse import Cache, _scale
from test_gpu_tables import _case, _dev, _eq, _list, _same_list

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _moves(got, want, what):
    got = got.cpu().tolist()
    assert got[:len(want)] == [list(x) for x in want] and all(x == [-1, -1] for x in got[len(want):]), what


@pytest.mark.parametrize("batch,width,block,spare,asked,n_moves", [
    (2, 4, 16, 10, 1.0, None), (2, 1, 1024, 0, 1.0, None), (7, 9, 4, 200, 0.8, None), (40, 30, 16, 900, 0.5, None),
    (40, 30, 16, 100, 0.5, None),            # the pool runs dry
    (40, 30, 16, 900, 0.5, 57),              # the list of pairs runs out
    (300, 6, 8, 2000, 0.7, None), (1000, 40, 16, 9000, 0.4, None), (4096, 3, 1, 5000, 0.6, None), (5, 700, 2, 5000, 0.9, None), (3, 5, 16, 40, 1.0, 0)])
def test_fork_against_the_oracle(batch, width, block, spare, asked, n_moves):
    for seed in range(3):
        print(f"fork batch={batch} width={width} block={block} spare={spare} n_moves={n_moves} seed={seed}", flush=True)
        rng = np.random.default_rng(seed + 11)
        table, lens, free = _case(rng, batch, width, block, spare)
        empty = rng.random(batch) < asked
        for b in np.flatnonzero(empty):
            free.back([x for x in table[b] if x >= 0])
            table[b], lens[b] = -1, 0
        source = np.where(rng.random(batch) < 0.9, rng.integers(-2, batch + 2, batch), np.arange(batch))   # some of themselves, of empty rows, of none
        if batch > 6:                        # entries outside the pool, lengths that are none
            full = np.flatnonzero(lens > 2 * block)
            if len(full):
                table[full[0], 1] = 1 << 25
                table[full[-1], 0] = -1
            lens[batch // 2] = -4
            lens[batch // 3] = width * block + 1 if batch % 2 else lens[batch // 3]
            free.stack = [x for x in free.stack]
        n = n_moves if n_moves is not None else int(sum(-(-max(int(lens[s]), 0) // block) for s in source if 0 <= s < batch)) + 3
        t, l, f = _dev(table), _dev(lens), _list(free)
        moves, granted = ckv.paged_fork(t, l, _dev(source), f, block, n)
        torch.cuda.synchronize()
        want, ok = po.fork(table, lens, source, free, block, n)
        _eq(granted, ok, "granted")
        _moves(moves, want, "moves")
        _eq(t, table, "table")
        _eq(l, lens, "lens")
        _same_list(f, free, "free list")


def test_fork_is_taken_back_by_a_trim():
    rng = np.random.default_rng(5)
    table, lens, free = _case(rng, 20, 12, 8, 300)
    lens[::2], before = 0, None
    for b in range(0, 20, 2):
        free.back([x for x in table[b] if x >= 0])
        table[b] = -1
    t, l, f = _dev(table), _dev(lens), _list(free)
    before = [x.clone() for x in (t, l, f)]
    moves, granted = ckv.paged_fork(t, l, _dev([b + 1 if b % 2 == 0 else -1 for b in range(20)]), f, 8, 300)
    assert granted.cpu().tolist() == [1, 0] * 10 and int((moves[:, 0] >= 0).sum()) == int(before[2][0] - f[0]) > 0
    ckv.paged_trim(t, l, before[1], f, 8)
    assert all(torch.equal(a, b) for a, b in zip((t, l, f), before))


@pytest.mark.parametrize("batch,width,block,spare,n_moves", [
    (1, 4, 16, 10, None), (1, 1, 1, 0, None), (6, 9, 4, 31, None), (6, 9, 4, 32, 3), (33, 70, 32, 700, None), (33, 70, 32, 30000, None),
    (33, 70, 32, 700, 0), (300, 6, 8, 64, None), (4096, 3, 2, 2500, None), (5, 900, 1, 70000, 333)])
def test_compact_against_the_oracle(batch, width, block, spare, n_moves):
    for seed in range(3):
        print(f"compact batch={batch} width={width} block={block} spare={spare} n_moves={n_moves} seed={seed}", flush=True)
        rng = np.random.default_rng(seed + 3)
        table, lens, free = _case(rng, batch, width, block, spare)
        for x in free.stack[:len(free.stack) // 5]:              # blocks of other tables
            free.stack.remove(x)
            free.dealt.add(x)
        if batch > 5:
            full = np.flatnonzero(lens > 2 * block)
            if len(full) > 2:
                table[full[0], 0], table[full[1], 1] = -1, free.n_blocks
                table[full[-1], 0] = table[full[-1], 1]          # a block that two entries name
            table[0, -1] = table[full[0], 1] if len(full) else -1   # behind the tokens: not looked at
            lens[0] = min(lens[0], (width - 1) * block)
            lens[1] = -7
        n = n_moves if n_moves is not None else free.n_blocks + 2
        t, l, f = _dev(table), _dev(lens), _list(free)
        moves, extent = ckv.paged_compact(t, l, f, block, n)
        torch.cuda.synchronize()
        want, top = po.compact(table, lens, free, block, n)
        _moves(moves, want, "moves")
        assert extent.tolist() == [top]
        _eq(t, table, "table")
        _eq(l, lens, "lens")
        _same_list(f, free, "free list")
        assert (f[4 + len(free.stack):4 + free.n_blocks] == -1).all()


@pytest.mark.parametrize("dtype,heads,dim,block,blocks,n", [
    ("bf16", 8, 128, 16, 40, 17), ("bf16", 1, 64, 1, 300, 131), ("f32", 3, 32, 4, 90, 44), ("bf16", 2, 64, 1024, 5, 2), ("f32", 5, 4, 8, 70, 30),
    ("bf16", 7, 128, 32, 11, 5)])
@pytest.mark.parametrize("with_deg,with_bounds", [(True, True), (False, False), (True, False)])
def test_copy(dtype, heads, dim, block, blocks, n, with_deg, with_bounds):
    print(f"copy {dtype} {heads}x{dim} block {block} of {blocks}", flush=True)
    g = torch.Generator().manual_seed(3)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pools = [torch.randn(blocks, heads, block, dim, generator=g).to(dt) for _ in range(2)]
    pools.append(torch.randint(1, 99, (blocks, heads, block), generator=g, dtype=torch.int32) if with_deg else None)
    pools.append(torch.randn(blocks, heads, 2, dim, generator=g).to(dt) if with_bounds else None)
    pools.append(torch.randint(1, 99, (blocks, heads), generator=g, dtype=torch.int32) if with_bounds else None)
    order = torch.randperm(blocks, generator=g)
    pairs = torch.stack([order[torch.randint(0, blocks - n, (n,), generator=g)], order[blocks - n:]], 1)    # (a source serves several)
    some = torch.tensor([[-1, -1], [int(pairs[0, 0]), blocks], [blocks + 5, int(order[0])], [-3, int(order[0])], [int(order[0])] * 2])
    moves = torch.cat([pairs, some])[torch.randperm(n + 5, generator=g)].to(torch.int32).to(DEV)
    dev = [None if p is None else p.to(DEV) for p in pools]
    ckv.paged_copy(moves, *dev)
    torch.cuda.synchronize()
    for p, d in zip(pools, dev):
        if p is not None:
            p[pairs[:, 1]] = p[pairs[:, 0]]
            assert torch.equal(p, d.cpu())
    ckv.paged_copy(moves[:0], *dev)


def test_copy_behind_32_bits():
    """Pages on either side of 4 GiB of a pool."""
    blocks = (1 << 32) // (8 * 16 * 128 * 2) + 40
    K, V = (torch.zeros((blocks, 8, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    K[blocks - 1], V[blocks - 1], K[3], V[3] = 1.0, 2.0, 3.0, 4.0
    ckv.paged_copy(_dev([[blocks - 1, 5], [3, blocks - 2], [3, blocks - 30]]), K, V)
    assert (K[5] == 1).all() and (V[5] == 2).all()
    for b in (blocks - 2, blocks - 30):
        assert (K[b] == 3).all() and (V[b] == 4).all()
    assert not K[6].any() and not K[4].any() and not K[blocks - 3].any()


def test_recorded_forks_compactions_and_copies():
    """fork, copy, trim, compact, copy as one graph, replayed on inputs that change; every replay against the eager calls."""
    block, heads, dim, batch, width = 8, 2, 64, 12, 10
    rng = np.random.default_rng(9)
    table, lens, free = _case(rng, batch, width, block, 200)
    for b in range(0, batch, 2):
        free.back([x for x in table[b] if x >= 0])
        table[b], lens[b] = -1, 0
    nb = free.n_blocks
    K = torch.randn(nb, heads, block, dim, device=DEV).to(torch.bfloat16)
    start = [_dev(table), _dev(lens), _list(free), K, K + 1, torch.ones(nb, heads, block, dtype=torch.int32, device=DEV)]
    source = _dev(np.zeros(batch))
    cut = start[1].clone()
    ws = torch.empty(ckv.paged_compact_workspace(nb), dtype=torch.uint8, device=DEV)
    outs = lambda: ((_dev(np.zeros((nb, 2))), _dev(np.zeros(batch))), (_dev(np.zeros((nb, 2))), _dev([0])))

    def calls(s, out):
        (moves, granted), (down, extent) = out
        ckv.paged_fork(s[0], s[1], source, s[2], block, nb, out=(moves, granted))
        ckv.paged_copy(moves, s[3], s[4], s[5])
        ckv.paged_trim(s[0], s[1], cut, s[2], block)
        ckv.paged_compact(s[0], s[1], s[2], block, nb, out=(down, extent), workspace=ws)
        ckv.paged_copy(down, s[3], s[4], s[5])

    state, out = [x.clone() for x in start], outs()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        calls(state, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls(state, out)
    torch.cuda.synchronize()
    for step in range(4):
        source.copy_(_dev([(b + 1 + 2 * step) % batch if b % 2 == 0 else -1 for b in range(batch)]))
        cut.copy_(_dev([max(int(x) - 3 * (i % 4) * step, 0) if x else 5 * step * (i % 3) for i, x in enumerate(lens)]))
        want, want_out = [x.clone() for x in start], outs()
        calls(want, want_out)
        for x, y in zip(state, start):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state + [t for o in out for t in o], want + [t for o in want_out for t in o]):
            assert torch.equal(x, y), step


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_serving_run(dtype):
    """Two prompts; each forked twice, the forks continued by different tokens; one family ends, the pool is compacted, and every row that is
    left still answers as its own keys and values say."""
    block, heads, G, dim, batch, width = 16, 2, 4, 64, 6, 12
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(17)
    nb = 90
    K, V = (torch.full((nb, heads, block, dim), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    deg = torch.full((nb, heads, block), -7, dtype=torch.int32, device=DEV)
    bounds, mass = torch.zeros((nb, heads, 2, dim), dtype=dt, device=DEV), torch.zeros((nb, heads), dtype=torch.int32, device=DEV)
    table, lens, free = _dev(np.full((batch, width), -1)), _dev(np.zeros(batch)), ckv.paged_free_list(nb)
    text = [[] for _ in range(batch)]        # (key, value) rows of every sequence

    def extend(new):
        rows = sum(new)
        qkv = torch.randn(rows + 2, (G + 2) * heads, dim, generator=g).to(dt)
        slots, starts, granted = ckv.paged_reserve(table, lens, _dev(new), free, block, rows + 2)
        assert granted.tolist() == [1] * batch
        dev = qkv.to(DEV)
        q, k, v = dev[:, :G * heads], dev[:, G * heads:(G + 1) * heads], dev[:, (G + 1) * heads:]
        ckv.paged_write(k, v, slots, K, V, deg)
        o = ckv.paged_chunk_attn(q, K, V, deg, table, lens, starts, width * block)
        at = 0
        for b, n in enumerate(new):
            for i in range(at, at + n):
                text[b].append((qkv[i, G * heads:(G + 1) * heads], qkv[i, (G + 1) * heads:]))
            at += n
        check(o, qkv[:, :G * heads], _starts(new), new)

    def check(o, q, starts, new):
        for b, n in enumerate(new):
            if not n:
                continue
            one = Cache(0, [len(text[b])], heads, dim, block, dtype, False, spare=0, room=0)
            for t, (kr, vr) in enumerate(text[b]):
                blk = int(one.table[0, t // block])
                one.K[blk, :, t % block], one.V[blk, :, t % block] = kr, vr
            want, bound = _oracle(one, q[starts[b]:starts[b + 1]], [n], [0, n], True, _scale(dim))
            _close(o[starts[b]:starts[b + 1]], want, bound, dt, f"sequence {b}")

    extend([70, 0, 0, 101, 0, 0])
    moves, granted = ckv.paged_fork(table, lens, _dev([-1, 0, 0, -1, 3, 3]), free, block, 40)
    assert granted.tolist() == [0, 1, 1, 0, 1, 1]
    ckv.paged_copy(moves, K, V, deg, bounds, mass)
    for b, f in ((1, 0), (2, 0), (4, 3), (5, 3)):
        text[b] = list(text[f])
    extend([0, 5, 1, 33, 17, 20])            # each goes on by itself, within blocks that were copied half full
    extend([1, 1, 1, 1, 1, 1])
    ckv.paged_trim(table, lens, _dev([0, 0, 0, 500, 500, 110]), free, block)
    for b in range(3):
        text[b] = []
    text[5] = text[5][:110]
    moves, extent = ckv.paged_compact(table, lens, free, block, 60)
    ckv.paged_copy(moves, K, V, deg)
    used = sum(-(-len(x) // block) for x in text)
    assert extent.tolist() == [used] and int((moves[:, 0] >= 0).sum()) > 0 and int(free[0]) == nb - used
    assert sorted(x for x in table.flatten().tolist() if x >= 0) == list(range(used))
    extend([3, 0, 40, 2, 1, 7])
    q = torch.randn(batch, G * heads, dim, generator=g).to(dt)
    some = [0, 2, 3, 4, 5]
    o = ckv.paged_decode_attn(q.to(DEV), K, V, deg, table, lens, width * block)
    c = ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, lens, _dev(range(batch + 1)), width * block)
    for b in some:
        a = f64(o[b]) - f64(c[b])
        assert np.abs(a).max() < 2.0**-5, "one token by either call"
