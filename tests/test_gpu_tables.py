"""Block tables, slot maps and ragged writes on the GPU, against the oracle's one request after the other: whole numbers and
copies, so everything has to be equal."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _dev(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).to(DEV)


def _case(rng, batch, width, block, spare, full=0.7):
    """(table, lens, FreeList) of a cache in use, its pool dealt in random order."""
    lens = np.where(rng.random(batch) < 0.2, 0, rng.integers(0, int(width * block * full) + 1, batch))
    need = -(-lens // block)
    order = rng.permutation(max(int(need.sum()) + spare, 1))         # (a pool has a block)
    table, at = np.full((batch, width), -1), 0
    for b in range(batch):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    return table, lens, po.FreeList(len(order), order[at:])


def _list(free):
    """The free list of the library for the oracle's; what is behind the stack is random."""
    t = ckv.paged_free_list(free.n_blocks)
    marks = np.full(free.n_blocks, -1)
    marks[list(free.dealt)] = 2**31 - 1
    t[0] = len(free.stack)
    t[4:4 + len(free.stack)] = _dev(free.stack)
    t[4 + free.n_blocks:] = _dev(marks)
    return t


def _same_list(got, free, what):
    got = got.cpu().numpy()
    marks = np.full(free.n_blocks, -1)
    marks[list(free.dealt)] = 2**31 - 1
    assert got[0] == len(free.stack) and not got[1:4].any(), what
    assert got[4:4 + got[0]].tolist() == free.stack, what
    assert np.array_equal(got[4 + free.n_blocks:], marks), what


def _eq(got, want, what):
    assert torch.equal(got.cpu().to(torch.int64), torch.as_tensor(np.asarray(want), dtype=torch.int64)), what


@pytest.mark.parametrize("batch,width,block,spare,new,n_slots", [
    (1, 4, 16, 10, 1, None), (1, 1, 1, 0, 1, None), (1, 1, 1024, 1, 1024, None), (7, 9, 4, 60, 20, None), (64, 20, 16, 64, 1, None),
    (64, 20, 16, 9, 1, None),                # the pool runs dry
    (33, 70, 32, 3000, 700, None),           # prompts: more slots than a workgroup takes
    (33, 70, 32, 400, 700, None), (300, 6, 8, 900, 30, 2100),     # the slot map runs out
    (257, 3, 16, 0, 5, None), (4096, 2, 16, 3000, 9, None), (1000, 40, 16, 4000, 60, None), (5, 3, 2, 30, 0, 0), (6, 5, 16, 3, 9, 1)])
def test_reserve_against_the_oracle(batch, width, block, spare, new, n_slots):
    print(f"reserve batch={batch} width={width} block={block} spare={spare} new={new}", flush=True)
    rng = np.random.default_rng(batch * 1000 + width)
    for step in range(3):
        table, lens, free = _case(rng, batch, width, block, spare)
        n_new = rng.integers(0 if step else 1, new + 1, batch) if new else np.zeros(batch, dtype=np.int64)
        if step == 2:                        # odd requests among them
            n_new[rng.random(batch) < 0.1] = -5
            n_new[rng.random(batch) < 0.05] = 2**31 - 1
            lens[rng.random(batch) < 0.05] = -3
            table[rng.random(table.shape) < 0.05] = 2**30
        total = int(np.clip(n_new, 0, new).sum())
        slots_n = (total if n_slots is None else n_slots) + (5 if step == 1 else 0)
        t, l, f = _dev(table), _dev(lens), _list(free)
        slots, starts, ok = ckv.paged_reserve(t, l, _dev(n_new), f, block, slots_n)
        want = po.reserve(table, lens, n_new, free, block, slots_n)
        for a, b, what in ((slots, want[0], "slots"), (starts, want[1], "starts"), (ok, want[2], "granted"), (t, table, "table"), (l, lens, "lens")):
            _eq(a, b, (step, what))
        _same_list(f, free, step)


@pytest.mark.parametrize("batch,width,block,spare", [(1, 3, 16, 2), (9, 30, 4, 11), (64, 700, 16, 90), (4096, 3, 8, 0), (3, 9000, 1, 5), (2000, 12, 16, 4)])
def test_trim_against_the_oracle(batch, width, block, spare):
    print(f"trim batch={batch} width={width} block={block}", flush=True)
    rng = np.random.default_rng(batch + width)
    for step in range(3):
        table, lens, free = _case(rng, batch, width, block, spare, full=1.0)
        cut = rng.integers(-1, lens + 3)
        if step == 1:
            cut[:] = 0
        if step == 2:                        # entries outside the pool, blocks that are free, the same block twice
            table[rng.random(table.shape) < 0.05] = 2**30
            table[rng.random(table.shape) < 0.05] = -1
            if free.stack:
                table[rng.random(table.shape) < 0.05] = free.stack[0]
            table[rng.random(table.shape) < 0.05] = int(table[0, 0])
            lens[rng.random(batch) < 0.05] = 2**31 - 1       # (longer than its row)
        t, l, f = _dev(table), _dev(lens), _list(free)
        ckv.paged_trim(t, l, _dev(cut), f, block)
        po.trim(table, lens, cut, free, block)
        _eq(t, table, step)
        _eq(l, lens, step)
        _same_list(f, free, step)


def test_a_reservation_taken_back_leaves_every_word_as_it_was():
    rng = np.random.default_rng(3)
    table, lens, free = _case(rng, 200, 30, 16, 500)
    t, l, f = _dev(table), _dev(lens), _list(free)
    t0, l0, f0 = t.clone(), l.clone(), f.clone()
    for new in (1, 40, 0):
        _, _, ok = ckv.paged_reserve(t, l, _dev(rng.integers(0, new + 1, 200)), f, 16, 200 * 40)
        assert new == 0 or not torch.equal(l, l0)
        ckv.paged_trim(t, l, l0, f, 16)
        torch.cuda.synchronize()
        assert torch.equal(t, t0) and torch.equal(l, l0) and torch.equal(f, f0)


@pytest.mark.parametrize("n", [0, 1, 5, 4096, 10001])
def test_free_against_the_oracle(n):
    rng = np.random.default_rng(n)
    table, lens, free = _case(rng, 8, 2000, 4, 40)
    f = _list(free)
    ids = rng.choice(np.concatenate([table.flatten(), [-1, -7, free.n_blocks, 2**30], free.stack]), n)    # (blocks come up twice)
    ckv.paged_free(_dev(ids), f)
    free.back(ids)
    _same_list(f, free, n)


@pytest.mark.parametrize("dtype,heads,dim,block,n,layout", [
    ("bf16", 8, 128, 16, 64, "qkv"), ("bf16", 8, 128, 16, 3001, "qkv"), ("f32", 2, 64, 32, 77, "qkv"), ("bf16", 1, 64, 1, 1, "plain"),
    ("bf16", 3, 8, 8, 500, "plain"), ("f32", 5, 36, 4, 100, "heads_first"), ("bf16", 40, 256, 16, 9, "plain"), ("f32", 1, 4, 2, 2000, "qkv")])
def test_write_against_indexing(dtype, heads, dim, block, n, layout):
    print(f"write {dtype} heads={heads} dim={dim} block={block} n={n} {layout}", flush=True)
    g = torch.Generator().manual_seed(n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda *s: torch.randn(s, generator=g).to(dt)
    if layout == "qkv":
        x = rnd(n, 3 * heads + 1, dim)
        k, v = x[:, heads:2 * heads], x[:, 2 * heads:3 * heads]
    elif layout == "heads_first":
        k, v = rnd(heads, n, dim).transpose(0, 1), rnd(heads, n, dim).transpose(0, 1)
    else:
        k, v = rnd(n, heads, dim), rnd(n, heads, dim)
    n_blocks = n // block + 3
    K, V, deg = rnd(n_blocks, heads, block, dim), rnd(n_blocks, heads, block, dim), torch.randint(5, 9, (n_blocks, heads, block), generator=g, dtype=torch.int32)
    slots = torch.randperm(n_blocks * block, generator=g)[:n].to(torch.int32)
    if n > 5:
        slots[2], slots[3], slots[5] = -1, n_blocks * block, 2**31 - 1
    dv = [y.to(DEV) for y in (K, V, deg)]
    if layout == "qkv":
        x_d = x.to(DEV)
        kd, vd = x_d[:, heads:2 * heads], x_d[:, 2 * heads:3 * heads]
    elif layout == "heads_first":
        kd, vd = (y.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) for y in (k, v))
    else:
        kd, vd = k.to(DEV), v.to(DEV)
    for with_deg in (True, False):
        Kd, Vd, dd = (y.clone() for y in dv)
        ckv.paged_write(kd, vd, slots.to(DEV), Kd, Vd, dd if with_deg else None)
        wK, wV, wd = K.clone(), V.clone(), deg.clone()
        for i, s in enumerate(slots.tolist()):
            if 0 <= s < n_blocks * block:
                wK[s // block, :, s % block], wV[s // block, :, s % block] = k[i], v[i]
                if with_deg:
                    wd[s // block, :, s % block] = 1
        torch.cuda.synchronize()
        assert torch.equal(Kd.cpu(), wK) and torch.equal(Vd.cpu(), wV) and torch.equal(dd.cpu(), wd)


def test_calls_by_ctypes_and_by_the_binding_agree(monkeypatch):
    class Never:
        def __getattr__(self, name):
            return lambda *a: None
    rng = np.random.default_rng(8)
    table, lens, free = _case(rng, 40, 12, 16, 60)
    n_new = _dev(rng.integers(0, 40, 40))
    real, outs, took = ckv._binding(), [], []
    for module in (real, Never()):
        monkeypatch.setattr(ckv, "_native", module)
        t, l, f = _dev(table), _dev(lens), _list(free)
        out = tuple(torch.zeros(n, dtype=torch.int32, device=DEV) for n in (1600, 41, 40))
        got = ckv.paged_reserve(t, l, n_new, f, 16, 1600, out=out)
        k = torch.arange(1600 * 2 * 64, device=DEV).remainder(97).to(torch.bfloat16).view(1600, 2, 64)
        K, V = (torch.zeros((free.n_blocks, 2, 16, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ckv.paged_write(k, k, got[0], K, V)
        grown = l.clone()
        ckv.paged_trim(t, l, _dev(lens // 2), f, 16)
        outs.append([*got, grown, t, l, f, K, V])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_steps_recorded_into_a_graph():
    """Reservations and trims recorded once and replayed: lengths, tables and the free list move on as in the oracle."""
    rng = np.random.default_rng(5)
    table, lens, free = _case(rng, 50, 40, 16, 300, full=0.3)
    t, l, f = _dev(table), _dev(lens), _list(free)
    n_new, cut = torch.ones(50, dtype=torch.int32, device=DEV), torch.full((50,), -1, dtype=torch.int32, device=DEV)
    out = tuple(torch.zeros(n, dtype=torch.int32, device=DEV) for n in (2048, 51, 50))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    ckv.paged_reserve(t, l, torch.zeros_like(n_new), f, 16, 2048, out=out)       # (kernels loaded before the capture)
    ckv.paged_trim(t, l, cut, f, 16)
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ckv.paged_reserve(t, l, n_new, f, 16, 2048, out=out)
        ckv.paged_trim(t, l, cut, f, 16)
    for rep in range(6):
        fresh, back = rng.integers(0, 40, 50), np.where(rng.random(50) < 0.3, 0, -1)
        n_new.copy_(_dev(fresh))
        cut.copy_(_dev(back))
        graph.replay()
        torch.cuda.synchronize()
        want = po.reserve(table, lens, fresh, free, 16, 2048)
        po.trim(table, lens, back, free, 16)
        for a, b, what in zip((*out, t, l), (*want, table, lens), ("slots", "starts", "granted", "table", "lens")):
            _eq(a, b, (rep, what))
        _same_list(f, free, rep)
