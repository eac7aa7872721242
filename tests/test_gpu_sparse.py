"""Block bounds, block selection and sparse decode attention on the GPU against the oracle: bounds and selections have to be
equal, attention within a tolerance that follows from its arithmetic."""
import numpy as np
import pytest
import torch

import oracle
import paper_2506_11418_amd as ckv
from oracle import paged_oracle as po
from parity_util import f64, i64

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Cache:
    """A pool whose blocks are dealt in random order to sequences of the given lengths; NaN in every row no token has."""

    def __init__(self, seed, lens, heads, dim, block, dtype="bf16", degrees=True, spare=3, room=2):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.dim, self.block, self.dtype = list(lens), heads, dim, block, DT[dtype]
        need = [-(-n // block) for n in self.lens]
        self.n_blocks = sum(need) + spare
        order = torch.randperm(self.n_blocks, generator=g).tolist()
        self.table = torch.full((len(self.lens), max(need) + room), -1, dtype=torch.int32)
        shape = (self.n_blocks, heads, block)
        self.K, self.V = (torch.full(shape + (dim,), float("nan"), dtype=self.dtype) for _ in range(2))
        self.deg = torch.full(shape, -7, dtype=torch.int32)
        loud = torch.ones(heads, 1, dim)
        loud[:, :, torch.randperm(dim, generator=g)[:dim // 32]] = 10.0
        at = 0
        for b, n in enumerate(self.lens):
            for i in range(need[b]):
                blk, rows = order[at], min(block, n - i * block)
                at += 1
                self.table[b, i] = blk
                near = torch.randn(heads, 1, dim, generator=g) * 0.9 + torch.randn(heads, rows, dim, generator=g) * 0.45
                self.K[blk, :, :rows] = (near * loud).to(self.dtype)
                self.V[blk, :, :rows] = torch.randn(heads, rows, dim, generator=g).to(self.dtype)
                self.deg[blk, :, :rows] = torch.randint(1, 9, (heads, rows), generator=g, dtype=torch.int32) if degrees else 1
        self.degrees = degrees

    def gpu(self):
        return self.K.to(DEV), self.V.to(DEV), self.deg.to(DEV) if self.degrees else None, self.table.to(DEV), _dev(self.lens)

    def want_bounds(self, bounds, mass, since=None, max_new=1 << 30):
        """bounds, mass (host) with the touched blocks filled in from their definition."""
        for b, n in enumerate(self.lens):
            s = 0 if since is None else max(int(since[b]), 0)
            for i in range(s // self.block, -(-min(n, s + max_new) // self.block) if min(n, s + max_new) > s else 0):
                blk = int(self.table[b, i])
                if not 0 <= blk < self.n_blocks:
                    continue
                rows = min(self.block, n - i * self.block)
                for h in range(self.heads):
                    lo, hi, m = po.bounds(f64(self.K[blk, h, :rows]), i64(self.deg[blk, h, :rows]))
                    bounds[blk, h, 0], bounds[blk, h, 1] = torch.from_numpy(lo).to(self.dtype), torch.from_numpy(hi).to(self.dtype)
                    mass[blk, h] = m
        return bounds, mass

    def want_select(self, q, bounds, mass, max_len, n_select, n_sink, n_recent, scale):
        """(sel, sel_lens, positions per (sequence, head)) from host bounds."""
        G = q.shape[1] // self.heads
        sel = np.full((len(self.lens), self.heads, n_select), -1)
        tokens, picked = np.zeros(sel.shape[:2], dtype=np.int64), {}
        for b, n in enumerate(self.lens):
            n = max(min(n, max_len, self.table.shape[1] * self.block), 0)
            cols = -(-n // self.block)
            ids = i64(self.table[b, :cols])
            inside = (ids >= 0) & (ids < self.n_blocks)
            at = torch.from_numpy(np.where(inside, ids, 0))
            for h in range(self.heads):
                m = i64(mass[at, h])
                s = po.scores(f64(q[b, h * G:(h + 1) * G]), f64(bounds[at, h, 0]), f64(bounds[at, h, 1]), np.maximum(m, 1), scale)
                s = [x if ok else "out" for x, ok in zip(s.tolist(), inside & (m > 0))]
                pos = po.select(s, cols, n_select, n_sink, n_recent) if cols > n_select else list(range(cols))
                picked[b, h] = pos
                sel[b, h, :len(pos)] = [int(ids[i]) * self.heads + h if inside[i] else -1 for i in pos]
                tokens[b, h] = sum(min(self.block, n - i * self.block) for i in pos)
        return sel, tokens, picked


def _dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _queries(seed, batch, q_heads, dim, dtype):
    return torch.randn(batch, q_heads, dim, generator=torch.Generator().manual_seed(seed)).to(DT[dtype])


def _scale(dim):
    return float(np.float32(1.0) / np.sqrt(np.float32(dim)))


def _same(a, b):
    """Equal, NaN where NaN."""
    a, b = a.cpu(), b.cpu()
    return a.shape == b.shape and bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("dtype,heads,dim,block,lens,degrees", [
    ("bf16", 8, 128, 16, [1, 16, 17, 0, 500], True), ("bf16", 2, 64, 1, [1, 7, 40], True), ("bf16", 1, 128, 1024, [1, 1500, 1024], False),
    ("bf16", 3, 64, 64, [130, 63], False), ("bf16", 5, 128, 8, [77, 3], True), ("f32", 2, 32, 16, [33, 5], True),
    ("f32", 4, 64, 32, [100, 32, 1], False), ("f32", 1, 128, 4, [19], True), ("f32", 8, 128, 256, [600], True)])
def test_bounds_against_the_oracle(dtype, heads, dim, block, lens, degrees):
    print(f"bounds {dtype} heads={heads} dim={dim} block={block} lens={lens}", flush=True)
    c = Cache(7, lens, heads, dim, block, dtype, degrees)
    if degrees:                              # tokens of degree 0 and below do not count, a block of none has no bounds
        c.deg[c.deg > 6] = 0
        c.deg[int(c.table[-1, 0])] = -1
    c.table[0, -1] = 1 << 28                 # (behind the sequence)
    K, _, deg, table, n = c.gpu()
    shape = (c.n_blocks, heads, 2, dim)
    for since, max_new in ((None, max(lens)), ([max(x - 1, 0) for x in lens], 1), ([x // 2 for x in lens], 30), ([-5] * len(lens), 3),
                           ([x for x in lens], 10), ([0] * len(lens), 2**31 - 1)):
        bounds, mass = torch.full(shape, 3.0, dtype=c.dtype, device=DEV), torch.full(shape[:2], 5, dtype=torch.int32, device=DEV)
        wb, wm = c.want_bounds(bounds.cpu(), mass.cpu(), since, max_new)
        ckv.paged_bounds(K, deg, table, n, max_new, since=None if since is None else _dev(since), out=(bounds, mass))
        torch.cuda.synchronize()
        assert _same(bounds, wb) and torch.equal(mass.cpu(), wm), (since, max_new)


def test_bounds_of_keys_that_are_no_numbers():
    c = Cache(8, [40, 33], 2, 64, 16)
    blk = int(c.table[0, 0])
    c.K[blk, 0, 3, 5], c.K[blk, 0, 4, 6], c.K[blk, 1, 0, 0] = float("nan"), float("inf"), float("-inf")
    c.table[1, 1] = -1                       # an entry outside the pool is passed over
    K, _, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 40)
    torch.cuda.synchronize()
    wb, wm = c.want_bounds(torch.zeros(bounds.shape, dtype=c.dtype), torch.zeros(mass.shape, dtype=torch.int32))
    wb[blk, 0, :, 5] = float("nan")
    assert _same(bounds, wb) and torch.equal(mass.cpu(), wm)


CASES = [
    # dtype, heads, group, dim, block, lens, n_select, n_sink, n_recent, degrees
    ("bf16", 8, 4, 128, 16, [2050], 32, 1, 1, True), ("bf16", 2, 1, 128, 16, [1, 0, 17, 300, 5000], 4, 1, 1, True),
    ("bf16", 1, 8, 64, 8, [999, 1000, 1001], 20, 0, 0, True), ("bf16", 4, 2, 64, 64, [4096, 65, 3000], 7, 2, 3, False),
    ("bf16", 3, 8, 128, 1, [257, 64], 63, 5, 9, True), ("f32", 4, 2, 64, 32, [9001, 4500], 48, 1, 1, True),
    ("f32", 1, 4, 32, 16, [700, 33], 1, 0, 1, False), ("f32", 2, 8, 128, 16, [1111], 16, 1, 0, True), ("f32", 2, 1, 32, 4, [50], 12, 12, 0, True),
    ("bf16", 1, 2, 128, 16, [70000], 256, 1, 1, False), ("bf16", 33, 4, 64, 16, [400, 200], 9, 1, 1, True), ("bf16", 1, 1, 64, 2, [30011], 999, 3, 3, True),
    # long rows: cut into segments, few and many kept, short sequences among them; and one wanted too many of for that
    ("f32", 2, 2, 32, 1, [20000, 9, 2049, 4096], 7, 2, 0, False), ("bf16", 1, 4, 64, 1, [33333, 15000], 514, 1, 1, True),
    ("f32", 1, 1, 32, 1, [40001], 600, 0, 1, False), ("f32", 1, 1, 32, 2, [30000], 6, 4, 2, True),
]


@pytest.mark.parametrize("dtype,heads,group,dim,block,lens,n_select,n_sink,n_recent,degrees", CASES)
def test_selection_and_attention_against_the_oracle(dtype, heads, group, dim, block, lens, n_select, n_sink, n_recent, degrees):
    print(f"sparse {dtype} heads={heads}x{group} dim={dim} block={block} lens={lens} select={n_select}", flush=True)
    c = Cache(11, lens, heads, dim, block, dtype, degrees)
    q = _queries(5, len(lens), heads * group, dim, dtype)
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, max(max(lens), 1))
    for max_len, scale in ((max(lens), 0.0), (max(max(lens) // 2, 1), 0.3)):
        real = np.float32(scale).item() if scale else _scale(dim)
        sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, max_len, n_select, block, n_sink, n_recent, scale=scale)
        o = ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, scale=scale, out_dtype=torch.float32)
        torch.cuda.synchronize()
        want, tokens, picked = c.want_select(q, bounds.cpu(), mass.cpu(), max_len, n_select, n_sink, n_recent, real)
        assert np.array_equal(i64(sel_lens), tokens)
        assert np.array_equal(i64(sel), want)
        _check_attention(c, q, o, picked, max_len, real)


def _check_attention(c, q, o, picked, max_len, scale):
    """Against Eq. 3 over the picked tokens in 64 bits.  A logit's fp32 sum over dim products (exact for bf16, one rounding each for
    fp32) is off by at most (dim + 8) 2^-24 sum |q k| scale, its logarithm and scaling by 2^-20; a weight by twice that relatively,
    and the fp32 sums over tokens by 2^-16 at most (slices of tiles of 16 tokens, added up in order): all against the largest
    value."""
    G = q.shape[1] // c.heads
    for (b, h), pos in picked.items():
        n = max(min(c.lens[b], max_len), 0)
        tok = [(int(c.table[b, i]), r) for i in pos for r in range(min(c.block, n - i * c.block)) if 0 <= int(c.table[b, i]) < c.n_blocks]
        tok = [(blk, r) for blk, r in tok if int(c.deg[blk, h, r]) > 0]
        got = f64(o[b, h * G:(h + 1) * G])
        if not tok:
            assert not got.any()
            continue
        at = tuple(torch.tensor(x) for x in zip(*tok))
        k, v, d = f64(c.K[at[0], h, at[1]]), f64(c.V[at[0], h, at[1]]), i64(c.deg[at[0], h, at[1]])
        qs = f64(q[b, h * G:(h + 1) * G])
        x = qs @ k.T * scale + np.log(d)
        w = np.exp(x - x.max(1, keepdims=True))
        ref = w @ v / w.sum(1, keepdims=True)
        off = (c.dim + 8) * 2.0**-24 * (np.abs(qs) @ np.abs(k).T).max() * scale + 2.0**-20
        step = 0.0 if o.dtype == torch.float32 else 2.0**-8
        assert (np.abs(got - ref) <= (2 * off + 2.0**-16) * np.abs(v).max() + step * np.abs(ref)).all(), (b, h, np.abs(got - ref).max(), off)


def test_every_block_selected_is_attention_over_the_whole_cache():
    c = Cache(12, [500, 31, 0, 1], 4, 128, 16)
    q = _queries(6, 4, 16, 128, "bf16").to(DEV)
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 500)
    for n_select in (32, 40):
        sel, sel_lens = ckv.paged_select(q, bounds, mass, table, n, 500, n_select, 16)
        o = ckv.paged_sparse_decode_attn(q, K, V, deg, sel, sel_lens, out_dtype=torch.float32)
        full = ckv.paged_decode_attn(q, K, V, deg, table, n, 500, out_dtype=torch.float32)
        torch.cuda.synchronize()
        assert sel_lens.tolist() == [[x] * 4 for x in c.lens] and bool((sel[2] == -1).all())
        _check_attention(c, q.cpu(), o, {(b, h): list(range(-(-x // 16))) for b, x in enumerate(c.lens) for h in range(4)}, 500, _scale(128))
        assert (o - full).abs().max() < 1e-4


def test_ranks_of_equal_missing_and_infinite_scores():
    """Equal blocks come in order; blocks whose bounds or query are not finite come first, those without mass or outside the pool
    last, and their tokens are masked."""
    c = Cache(13, [16 * 40, 16 * 40], 2, 64, 16, degrees=True)
    for i in range(5, 30):                   # equal blocks
        c.K[int(c.table[0, i])] = c.K[int(c.table[0, 5])]
        c.deg[int(c.table[0, i])] = c.deg[int(c.table[0, 5])]
    c.K[int(c.table[0, 33]), 0, 2, 7] = float("nan")
    c.K[int(c.table[0, 35]), 0, 2, 7] = float("inf")
    c.K[int(c.table[0, 36]), 0, 2, 7] = float("-inf")
    c.deg[int(c.table[0, 2])] = 0
    c.table[0, 3], c.table[0, 4] = -1, 1 << 29
    q = _queries(7, 2, 8, 64, "bf16")
    q[1, 5, 3] = float("inf")                # (its KV head selects in order of position)
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 640)
    for n_select in (1, 2, 5, 11, 33, 37, 38, 39):
        sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, 640, n_select, 16, n_sink=0, n_recent=1)
        torch.cuda.synchronize()
        want, tokens, _ = c.want_select(q, bounds.cpu(), mass.cpu(), 640, n_select, 0, 1, _scale(64))
        assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), tokens), n_select
    # without the keys that are no numbers, everything else selected: masked tokens leave the output finite
    c.K[int(c.table[0, 33]), 0, 2, 7] = c.K[int(c.table[0, 35]), 0, 2, 7] = c.K[int(c.table[0, 36]), 0, 2, 7] = 1.0
    q[1, 5, 3] = 1.0
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 640)
    sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, 640, 39, 16)
    o = ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, out_dtype=torch.float32)
    torch.cuda.synchronize()
    _, _, picked = c.want_select(q, bounds.cpu(), mass.cpu(), 640, 39, 1, 1, _scale(64))
    _check_attention(c, q, o, picked, 640, _scale(64))


@pytest.mark.parametrize("tokens,n_select", [(300, 40), (12000, 100), (12000, 300), (12000, 700)])
def test_ties_over_long_rows_go_to_the_lower_blocks(tokens, n_select):
    """Blocks of one token with few different keys: the cut falls among many equal scores, in every form the selection takes."""
    g = torch.Generator().manual_seed(n_select)
    some = torch.randn(5, 32, generator=g)
    c = Cache(15, [tokens, tokens // 3], 1, 32, 1, "f32", degrees=False)
    for b, n in enumerate(c.lens):
        c.K[c.table[b, :n].long(), 0, 0] = some[torch.randint(0, 5, (n,), generator=g)]
    q = _queries(10, 2, 2, 32, "f32")
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, tokens)
    for n_sink, n_recent in ((0, 0), (1, 1), (n_select, 0), (0, n_select)):
        sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, tokens, n_select, 1, n_sink, n_recent)
        torch.cuda.synchronize()
        want, count, _ = c.want_select(q, bounds.cpu(), mass.cpu(), tokens, n_select, n_sink, n_recent, _scale(32))
        assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), count), (n_sink, n_recent)


def test_outputs_of_the_cache_type_and_by_either_route(monkeypatch):
    class Never:
        def __getattr__(self, name):
            return lambda *a: None
    c = Cache(14, [3000, 123], 8, 128, 16)
    q = _queries(8, 2, 32, 128, "bf16")
    K, V, deg, table, n = c.gpu()
    real, outs = ckv._binding(), []
    for module in (real, Never()):
        monkeypatch.setattr(ckv, "_native", module)
        b = (torch.zeros(c.n_blocks, 8, 2, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(c.n_blocks, 8, dtype=torch.int32, device=DEV))
        ckv.paged_bounds(K, deg, table, n, 3000, out=b)
        out = tuple(torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((2, 8, 20), (2, 8)))
        ws = [torch.zeros(1 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]
        sel, sel_lens = ckv.paged_select(q.to(DEV), *b, table, n, 3000, 20, 16, out=out, workspace=ws[0])
        o = torch.zeros(2, 32, 128, dtype=torch.bfloat16, device=DEV)
        ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, out=o, workspace=ws[1])
        outs.append([*b, sel, sel_lens, o])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    _, _, picked = c.want_select(q, outs[0][0].cpu(), outs[0][1].cpu(), 3000, 20, 1, 1, _scale(128))
    _check_attention(c, q, outs[0][4], picked, 3000, _scale(128))


def test_workspaces_stay_inside_and_serve_calls_in_a_row():
    """One select and one attention workspace for calls of different shapes, sized for the largest: nothing behind them is
    written, and every call gives what it gives with workspaces of its own; also on another stream."""
    cs = [Cache(20, [1500, 700, 20], 8, 64, 16), Cache(21, [9000], 2, 64, 16), Cache(22, [64, 90, 3], 8, 64, 16)]
    sizes, calls = [0, 0], []
    for c in cs:
        q = _queries(9, len(c.lens), c.heads * 4, 64, "bf16").to(DEV)
        K, V, deg, table, n = c.gpu()
        b = ckv.paged_bounds(K, deg, table, n, max(c.lens))
        pl = ckv.paged_layout_of(K, table)
        sizes = [max(sizes[0], ckv.paged_select_workspace(pl, max(c.lens))), max(sizes[1], ckv.paged_sparse_decode_attn_workspace(pl, c.heads * 4, 24))]

        def call(ws=(None, None), q=q, b=b, table=table, n=n, K=K, V=V, deg=deg, c=c):
            sel, sel_lens = ckv.paged_select(q, *b, table, n, max(c.lens), 24, 16, workspace=ws[0])
            return sel, sel_lens, ckv.paged_sparse_decode_attn(q, K, V, deg, sel, sel_lens, workspace=ws[1])
        calls.append(call)
    held = [torch.full((s + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV) for s in sizes]
    for h, s in zip(held, sizes):
        h[:s] = 0
    want = [call() for call in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            for i in (0, 1, 2, 1, 0, 2, 0):
                got = calls[i]([h[:s] for h, s in zip(held, sizes)])
                torch.cuda.synchronize()
                assert all(torch.equal(x, y) for x, y in zip(got, want[i])), i
                assert all(bool((h[s:] == 0xA5).all()) for h, s in zip(held, sizes))


def test_a_serving_run_from_reservation_to_attention():
    """Prompts reserved, written and bounded; decode steps in one captured graph; two sequences compressed and their blocks given
    back; a finished one replaced: every step's slots, bounds, selection and attention against the oracle."""
    rng = np.random.default_rng(31)
    H, G, D, bs, batch, width, n_blocks, n_select = 4, 4, 128, 16, 5, 60, 200, 12
    g = torch.Generator().manual_seed(2)
    rows = lambda n: torch.randn(n, H, D, generator=g).to(torch.bfloat16)
    pool = lambda: torch.full((n_blocks, H, bs, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    K, V, deg = pool(), pool(), torch.zeros((n_blocks, H, bs), dtype=torch.int32, device=DEV)
    table, lens = torch.full((batch, width), -1, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    free = ckv.paged_free_list(n_blocks)
    bounds, mass = torch.zeros((n_blocks, H, 2, D), dtype=torch.bfloat16, device=DEV), torch.zeros((n_blocks, H), dtype=torch.int32, device=DEV)
    ofree, otable, olens = po.FreeList(n_blocks), np.full((batch, width), -1), np.zeros(batch, dtype=np.int64)

    def host(c=None):
        """The state on the GPU as a Cache."""
        c = Cache.__new__(Cache)
        c.lens, c.heads, c.dim, c.block, c.dtype, c.n_blocks, c.degrees = lens.tolist(), H, D, bs, torch.bfloat16, n_blocks, True
        c.table, c.K, c.V, c.deg = table.cpu(), K.cpu(), V.cpu(), deg.cpu()
        return c

    def admit(new):
        k, v = rows(int(sum(new))), rows(int(sum(new)))
        before = lens.clone()
        slots, starts, ok = ckv.paged_reserve(table, lens, _dev(new), free, bs, len(k) + 3)
        pad = torch.zeros(3, H, D, dtype=torch.bfloat16)
        ckv.paged_write(torch.cat([k, pad]).to(DEV), torch.cat([v, pad]).to(DEV), slots, K, V, deg)
        ckv.paged_bounds(K, deg, table, lens, max(new), since=before, out=(bounds, mass))
        want = po.reserve(otable, olens, new, ofree, bs, len(k) + 3)
        torch.cuda.synchronize()
        assert [x.tolist() for x in (slots, starts, ok)] == list(want) and min(want[2]) == 1
        assert np.array_equal(i64(table), otable) and np.array_equal(i64(lens), olens)
        for i, s in enumerate(want[0][:-3]):
            assert torch.equal(K[s // bs, :, s % bs].cpu(), k[i]) and torch.equal(V[s // bs, :, s % bs].cpu(), v[i])

    def check(q, sel, sel_lens, o):
        c = host()
        wb, wm = c.want_bounds(bounds.cpu(), mass.cpu())
        assert _same(bounds, wb) and torch.equal(mass.cpu(), wm)
        want, tokens, picked = c.want_select(q.cpu(), wb, wm, width * bs, n_select, 1, 1, _scale(D))
        assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), tokens)
        _check_attention(c, q.cpu(), o, picked, width * bs, _scale(D))

    admit([300, 17, 640, 1, 512])
    # a decode step, recorded: one token a sequence
    k1, v1, q = (torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((batch, H, D), (batch, H, D), (batch, H * G, D)))
    one, before = torch.ones(batch, dtype=torch.int32, device=DEV), torch.zeros_like(lens)
    out = tuple(torch.zeros(n, dtype=torch.int32, device=DEV) for n in (batch, batch + 1, batch))
    so = tuple(torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((batch, H, n_select), (batch, H)))
    o = torch.zeros(batch, H * G, D, dtype=torch.float32, device=DEV)
    pl = ckv.paged_layout_of(K, table)
    ws = torch.zeros(ckv.paged_select_workspace(pl, width * bs), dtype=torch.uint8, device=DEV)
    ws2 = torch.zeros(ckv.paged_sparse_decode_attn_workspace(pl, H * G, n_select), dtype=torch.uint8, device=DEV)

    def step():
        before.copy_(lens)
        ckv.paged_reserve(table, lens, one, free, bs, batch, out=out)
        ckv.paged_write(k1, v1, out[0], K, V, deg)
        ckv.paged_bounds(K, deg, table, lens, 1, since=before, out=(bounds, mass))
        ckv.paged_select(q, bounds, mass, table, lens, width * bs, n_select, bs, out=so, workspace=ws)
        ckv.paged_sparse_decode_attn(q, K, V, deg, *so, out=o, workspace=ws2)

    def advance(run):
        k1.copy_(rows(batch)); v1.copy_(rows(batch)); q.copy_(torch.randn(batch, H * G, D, generator=g))
        run()
        torch.cuda.synchronize()
        want = po.reserve(otable, olens, [1] * batch, ofree, bs, batch)
        assert out[0].tolist() == want[0] and out[2].tolist() == [1] * batch
        check(q, *so, o)

    advance(step)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(18):
        advance(graph.replay)
    # the two longest sequences are compressed in their pages, what they no longer need returns
    for b in (2, 4):
        n = int(lens[b])
        new, freed = ckv.paged_compress(K, V, deg, table[b:b + 1], n, 64, retain_ratio=0.5, lens=lens[b:b + 1])
        ckv.paged_free(freed, free)
        torch.cuda.synchronize()
        ofree.back(freed.flatten().tolist())
        otable[b, -(-new // bs):], olens[b] = -1, new
    ckv.paged_bounds(K, deg, table, lens, width * bs, out=(bounds, mass))
    advance(graph.replay)
    # sequence 0 has finished; another prompt takes its row
    cut = _dev([0, -1, -1, -1, -1])
    ckv.paged_trim(table, lens, cut, free, bs)
    po.trim(otable, olens, [0, -1, -1, -1, -1], ofree, bs)
    admit([777, 0, 0, 0, 0])
    for _ in range(3):
        advance(graph.replay)
    assert int(free[0]) == len(ofree.stack) and free[4:4 + len(ofree.stack)].tolist() == ofree.stack
