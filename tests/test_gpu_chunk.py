"""Attention of several new tokens over pages on the GPU against the oracle in 64 bits.

Bounds of an error, element by element, with A the weighted mean of |v| and u the rounding of a type (half a step): bf16 weights are
off by u each and so is their sum, 2 u A, and the output by u |o|; a logit by d relative weights the output by 2 d A, where d is
what fp32 sums of dim products, their scaling, the bias and 2^x leave: (dim + 8) 2^-24 times the largest sum of |q k| scale plus ln N, plus
2^-22; sums of n terms in fp32 by (n / 2 + 64) 2^-24 A, twice (numerator and denominator; two lanes share the terms)."""
import math

import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from oracle import paged_oracle as po
from parity_util import f64, i64
from test_gpu_sparse import Cache, _dev, _scale

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}


def _oracle(c, q, new, starts, causal, scale, max_len=1 << 30):
    """(o, bound) [rows, q_heads, dim]; rows of no sequence zero."""
    rows, q_heads, D = q.shape
    G = q_heads // c.heads
    want, bound = np.zeros((rows, q_heads, D)), np.zeros((rows, q_heads, D))
    for b, n in enumerate(c.lens):
        n = max(min(n, max_len, c.table.shape[1] * c.block), 0)
        lo, hi = starts[b], starts[b + 1]
        ids = i64(c.table[b, :-(-n // c.block)])
        inside = np.repeat((ids >= 0) & (ids < c.n_blocks), c.block)[:n]
        at = torch.from_numpy(np.where((ids >= 0) & (ids < c.n_blocks), ids, 0))
        seen = [n - (hi - lo) + i + 1 if causal else n for i in range(hi - lo)]
        for h in range(c.heads):
            k, v = (f64(p[at, h].reshape(-1, D)[:n]) for p in (c.K, c.V))
            deg = i64(c.deg[at, h].reshape(-1)[:n]) if c.degrees else np.ones(n, dtype=np.int64)
            deg = np.where(inside, deg, 0)
            heads = slice(h * G, (h + 1) * G)
            o, a, x = po.chunk_attention(f64(q[lo:hi, heads]), k, v, deg, seen, scale)
            d = (D + 8) * 2.0**-24 * (x * scale + math.log(max(deg.max(initial=1), 1)) + 1) + 2.0**-22
            u = 2 * U[q.dtype] if q.dtype == torch.bfloat16 else 0.0
            want[lo:hi, heads], bound[lo:hi, heads] = o, (u + 2 * d[..., None] + (n + 128) * 2.0**-24) * a
    return want, bound


def _close(got, want, bound, o_dtype, what=""):
    got = f64(got)
    ok = np.abs(got - want) <= (1 + 2.0**-8) * bound + U[o_dtype] * np.abs(want) + 1e-37
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all(), f"{what}: NaN at {np.argwhere(np.isnan(got) != nan)[:4].tolist()}"
    bad = ~(ok | nan)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]!r}, not {want[i]!r} (bound {bound[i]!r})")


def _queries(seed, rows, q_heads, dim, dtype):
    return torch.randn(rows, q_heads, dim, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _starts(new, lead=0):
    return [lead] + [lead + int(x) for x in np.cumsum(new)]


CASES = [
    # dtype, heads, group, dim, block, lens, new, degrees, causal
    ("bf16", 8, 4, 128, 16, [515], [33], True, True),
    ("bf16", 8, 4, 128, 16, [1, 64, 65, 127, 129], [1, 64, 1, 127, 3], True, True),
    ("bf16", 2, 1, 128, 16, [300, 0, 40, 200], [130, 0, 40, 129], False, True),
    ("bf16", 1, 8, 64, 8, [1000, 77], [17, 16], True, True),
    ("bf16", 4, 2, 64, 64, [2100], [65], False, True),
    ("bf16", 3, 4, 128, 1, [70, 3], [5, 3], True, True),
    ("bf16", 1, 2, 64, 1024, [1500, 1024], [200, 1], True, True),
    ("bf16", 2, 4, 128, 32, [40, 500], [31, 70], False, False),
    ("bf16", 2, 8, 64, 16, [0, 5, 130], [9, 40, 1], True, False),
    ("bf16", 2, 4, 64, 16, [20, 3], [30, 5], True, True),         # more new tokens than there are tokens
    ("f32", 2, 1, 32, 16, [33, 5], [33, 2], True, True),
    ("f32", 4, 2, 64, 32, [400, 32, 1], [70, 32, 1], False, True),
    ("f32", 1, 4, 128, 4, [219], [100], True, True),
    ("f32", 8, 8, 128, 256, [600], [3], True, False),
    ("f32", 1, 1, 64, 2, [31, 64, 33, 0, 1], [31, 1, 33, 2, 1], True, True),
]


@pytest.mark.parametrize("dtype,heads,group,dim,block,lens,new,degrees,causal", CASES)
def test_against_the_oracle(dtype, heads, group, dim, block, lens, new, degrees, causal):
    print(f"chunk {dtype} {heads}x{group} dim {dim} block {block} lens {lens} new {new} degrees {degrees} causal {causal}", flush=True)
    c = Cache(31, lens, heads, dim, block, dtype, degrees)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new)
    rows = starts[-1] + 3                                        # rows of no sequence behind
    q = _queries(5, rows, heads * group, dim, c.dtype)
    want, bound = _oracle(c, q, new, starts, causal, _scale(dim))
    for o_dtype in (c.dtype, torch.float32):
        out = torch.full(q.shape, 7.0, dtype=o_dtype, device=DEV)
        ws = torch.full((ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), heads * group, rows, max(lens) + 1),), 255,
                        dtype=torch.uint8, device=DEV)       # (whatever it holds)
        ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), max(lens) + 1, causal=causal, out=out, workspace=ws)
        torch.cuda.synchronize()
        assert (out[starts[-1]:] == 7.0).all()
        _close(out[:starts[-1]], want[:starts[-1]], bound[:starts[-1]], o_dtype)
        again = torch.zeros_like(out)
        ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), max(lens) + 1, causal=causal, out=again, workspace=ws)
        assert torch.equal(again[:starts[-1]], out[:starts[-1]])


@pytest.mark.parametrize("dtype,heads,group,dim,block,batch,most,new,degrees,causal", [
    ("bf16", 14, 8, 64, 16, 4, 1100, (450, 450), True, True), ("bf16", 32, 4, 128, 16, 60, 1200, (1, 1), False, True),
    ("f32", 32, 2, 64, 8, 50, 1300, (1, 3), True, True), ("bf16", 40, 1, 64, 32, 64, 700, (0, 2), False, False),
    ("bf16", 32, 4, 64, 16, 65, 900, (0, 3), True, True), ("bf16", 16, 2, 128, 16, 64, 511, (1, 90), True, True)])
def test_more_rows_than_the_chip_has_places(dtype, heads, group, dim, block, batch, most, new, degrees, causal):
    """Where the rows fill the chip several times over only the last of them are cut, or none."""
    rng = np.random.default_rng(batch)
    fresh = [int(x) for x in rng.integers(new[0], new[1] + 1, batch)]
    lens = [max(int(x), y) for x, y in zip(rng.integers(most // 2, most + 1, batch), fresh)]
    test_against_the_oracle(dtype, heads, group, dim, block, lens, fresh, degrees, causal)


@pytest.mark.parametrize("dtype,dim,causal,o_dtype", [("bf16", 64, True, torch.bfloat16), ("bf16", 128, False, torch.float32), ("f32", 32, True, torch.float32)])
def test_the_last_rows_of_many_are_cut(dtype, dim, causal, o_dtype):
    """Long turns that fill the chip several times over, with some rows out of each stretch of 64 tokens against the oracle."""
    lens, new, heads, G = [9700, 9001, 9200], [4200, 4203, 4201], 2, 8
    print(f"last rows {dtype} {dim} {causal}", flush=True)
    c = Cache(83, lens, heads, dim, 16, dtype, True)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new, lead=2)
    q = _queries(15, starts[-1], heads * G, dim, c.dtype)
    ws = torch.full((ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), heads * G, q.shape[0], 9700),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=o_dtype, device=DEV)
    ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), 9700, causal=causal, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert (out[:2] == 7.0).all()
    rng, scale = np.random.default_rng(2), _scale(dim)
    for b in range(3):
        rows = np.array([min(t + int(rng.integers(0, 64)), new[b] - 1) for t in range(0, new[b], 64)])
        ids, h = table[b, :-(-lens[b] // 16)].cpu().long(), int(rng.integers(0, heads))
        k, v, d = (p[ids, h].reshape(-1, p.shape[-1])[:lens[b]] for p in (c.K, c.V, c.deg[..., None]))
        at, cols = torch.from_numpy(starts[b] + rows), slice(h * G, (h + 1) * G)
        seen = lens[b] - new[b] + rows + 1 if causal else np.full(len(rows), lens[b])
        o, a, x = po.chunk_attention(f64(q[at, cols]), f64(k), f64(v), i64(d[:, 0]), seen, scale)
        e = (dim + 8) * 2.0**-24 * (x * scale + math.log(9)) + 2.0**-22
        u = 2 * U[c.dtype] if c.dtype == torch.bfloat16 else 0.0
        _close(out[at.to(DEV), cols], o, (u + 2 * e[..., None] + (lens[b] + 128) * 2.0**-24) * a, o_dtype, f"sequence {b}")
    again = torch.zeros_like(out)
    ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), 9700, causal=causal, out=again, workspace=ws)
    assert torch.equal(again[2:], out[2:])


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_tokens_that_are_not_seen_do_not_reach_a_row(dtype, dim):
    """Infinities and NaN in keys and values behind a row, in tokens of degree 0, in the rest of a page and under entries outside the pool."""
    print(f"masked {dtype} {dim}", flush=True)
    lens, new = [200, 90], [70, 90]
    c = Cache(40, lens, 2, dim, 16, dtype, True)
    hit = [int(c.table[0, 150 // 16]), int(c.table[1, 40 // 16])]
    for blk, off in ((hit[0], 150 % 16), (hit[1], 40 % 16)):       # seen from tokens 150 and 40 on
        c.V[blk, 0, off, 3] = float("inf")
        c.V[blk, 1, off, dim - 1] = float("nan")
        c.V[blk, 1, off, 0] = float("-inf")
    gone = int(c.table[0, 2])
    c.deg[gone, :, 5] = 0
    c.deg[gone, 0, 6] = -3
    c.K[gone, :, 5:7], c.V[gone, :, 5:7] = float("nan"), float("inf")
    c.deg[gone, 1, 6] = 0
    c.table[0, 4], c.table[1, 3] = -1, 1 << 20
    c.K[0], c.V[0] = float("nan"), float("nan")                  # (what stands in for an entry outside the pool)
    for b in range(2):
        for j in range(-(-lens[b] // 16)):
            assert int(c.table[b, j]) != 0, "block 0 belongs to a token of this seed"
    K, V, deg, table, n = c.gpu()
    starts = _starts(new)
    q = _queries(6, starts[-1], 8, dim, c.dtype)
    want, bound = _oracle(c, q, new, starts, True, _scale(dim))
    out = ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), 200)
    got = f64(out)
    fin = np.isfinite(want)
    assert (np.isfinite(got) == fin).all()
    assert fin[:20].all() and not fin[20:70, :4, 3].any()         # (row 20 of the first sequence is token 150)
    assert (got[20:70, :4, 3] == np.inf).all() and (got[20:70, 4:, 0] == -np.inf).all() and np.isnan(got[20:70, 4:, dim - 1]).all()
    _close(torch.from_numpy(np.where(fin, got, 0)), np.where(fin, want, 0), np.where(fin, bound, 0), c.dtype)


def test_logits_that_are_no_numbers():
    c = Cache(41, [100], 1, 64, 16, "bf16", False)
    blk, off = int(c.table[0, 5]), 10                            # token 90: seen from row 10 on
    c.K[blk, 0, off] = float("nan")
    K, V, deg, table, n = c.gpu()
    q = _queries(7, 20, 4, 64, c.dtype)
    q[3, 1, 0] = float("inf")
    want, bound = _oracle(c, q, [20], [0, 20], True, _scale(64))
    assert np.isnan(want[10:]).all() and np.isnan(want[3, 1]).all() and not np.isnan(want[:3]).any()
    _close(ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev([0, 20]), 100), want, bound, c.dtype)


def test_logits_far_apart_and_rows_that_see_late():
    """A maximum that rises by thousands from tile to tile, and falls; a first tile without a token that counts."""
    c = Cache(43, [700], 1, 64, 16, "bf16", True)
    for j in range(44):
        c.K[int(c.table[0, j])] *= [1.0, 40.0, 0.0, 300.0][j // 4 % 4] if j < 24 else 3.0
    c.deg[c.table[0, :5].long()] = 0
    c.K[torch.isnan(c.K)] = 0
    K, V, deg, table, n = c.gpu()
    q = _queries(8, 150, 2, 64, c.dtype)
    want, bound = _oracle(c, q, [150], [0, 150], True, 0.5)
    _close(ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev([0, 150]), 700, scale=0.5), want, bound, c.dtype)


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 40.0, 1e30])
def test_scales(scale):
    c = Cache(47, [90], 1, 64, 16, "f32", True)
    K, V, deg, table, n = c.gpu()
    q = _queries(9, 40, 2, 64, c.dtype)
    if scale > 100:                                              # (logits that fp32 holds)
        q = q * 1e-33
    want, bound = _oracle(c, q, [40], [0, 40], True, float(np.float32(scale)))
    _close(ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev([0, 40]), 90, scale=scale), want, bound, c.dtype)


def test_single_tokens_are_decode_attention():
    """One new token a sequence: what paged_decode_attn computes, within both bounds."""
    lens = [1, 33, 700, 64]
    c = Cache(53, lens, 2, 128, 16)
    K, V, deg, table, n = c.gpu()
    q = _queries(10, 4, 8, 128, c.dtype)
    want, bound = _oracle(c, q, [1] * 4, _starts([1] * 4), True, _scale(128))
    o = ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(_starts([1] * 4)), 700)
    _close(o, want, bound, c.dtype)
    _close(ckv.paged_decode_attn(q.to(DEV), K, V, deg, table, n, 700), want, 2 * bound, c.dtype)


def test_views_of_a_fused_projection_and_a_leading_row():
    """Queries with strides of their own; starts that do not begin at row 0; a length bound below the length."""
    c = Cache(59, [300, 50], 2, 64, 16)
    K, V, deg, table, n = c.gpu()
    qkv = _queries(11, 40, 12, 64, c.dtype)
    starts = [4, 24, 39]
    want, bound = _oracle(c, qkv[:, :8], [20, 15], starts, True, _scale(64), max_len=280)
    out = torch.full((40, 8, 64), 3.0, dtype=c.dtype, device=DEV)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    big = qkv.to(DEV)
    ckv.paged_chunk_attn(big[:, :8], K, V, deg, table, n, _dev(starts), 280, out=out, workspace=ws)
    _close(out[4:39], want[4:39], bound[4:39], c.dtype)
    assert (out[:4] == 3.0).all() and (out[39:] == 3.0).all()
    by_heads = big[:, :8].transpose(0, 1).contiguous().transpose(0, 1)        # heads outermost
    assert torch.equal(ckv.paged_chunk_attn(by_heads, K, V, deg, table, n, _dev(starts), 280), torch.where(out == 3.0, 0, out))


def test_many_sequences_and_empty_ones():
    """More sequences than a workgroup has threads, most without new tokens."""
    lens = [5 + i % 37 for i in range(600)]
    new = [(i % 5 == 0) * (1 + i % 3) for i in range(600)]
    c = Cache(61, lens, 1, 64, 16)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new)
    q = _queries(12, starts[-1], 4, 64, c.dtype)
    want, bound = _oracle(c, q, new, starts, True, _scale(64))
    _close(ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table, n, _dev(starts), 50), want, bound, c.dtype)


def test_a_pool_behind_32_bits():
    """Pages beyond 4 GiB of a pool."""
    heads, dim, block, blocks = 8, 128, 16, (1 << 32) // (8 * 16 * 128 * 2) + 40
    small = Cache(67, [100], heads, dim, block, spare=1)
    table = torch.where(small.table >= 0, small.table + (blocks - small.n_blocks), -1)
    K, V = (torch.zeros((blocks, heads, block, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    deg = torch.ones((blocks, heads, block), dtype=torch.int32, device=DEV)
    for pool, part in ((K, small.K), (V, small.V), (deg, small.deg)):
        pool[blocks - small.n_blocks:] = part.to(DEV)
    q = _queries(13, 9, 32, dim, torch.bfloat16)
    want, bound = _oracle(small, q, [9], [0, 9], True, _scale(dim))
    _close(ckv.paged_chunk_attn(q.to(DEV), K, V, deg, table.to(DEV), _dev([100]), _dev([0, 9]), 100), want, bound, torch.bfloat16)


def test_recorded_calls_that_share_a_workspace():
    """Two graphs on one stream and one workspace, replayed in turn with eager work between; lengths that change between replays."""
    c = Cache(71, [900, 40], 2, 64, 16)
    K, V, deg, table, n = c.gpu()
    q = _queries(14, 30, 8, 64, c.dtype).to(DEV)
    starts, lens = _dev([0, 10, 30]), n.clone()
    ws = torch.empty(ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), 8, 30, 900), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(q) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        for i, causal in enumerate((True, False)):
            call = lambda: ckv.paged_chunk_attn(q, K, V, deg, table, lens, starts, 900, causal=causal, out=outs[i], workspace=ws)
            call()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call()
            graphs.append(g)
    for step in range(4):
        lens.copy_(n - step * 3)
        want = [ckv.paged_chunk_attn(q, K, V, deg, table, lens, starts, 900, causal=x) for x in (True, False)]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]), step
