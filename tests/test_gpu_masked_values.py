"""Decode attention where the rows that do not count hold no numbers: table entries outside the pool (whose loads fall on row 0),
tokens of degree 0 and below, and the places behind the last token of a cache (whose loads fall on that token)."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_sparse import DEV, Cache, _check_attention, _queries, _scale

pytestmark = pytest.mark.gpu


def _without_block_0(c):
    """Block 0 changes places with one that no sequence has: its rows are NaN."""
    used = set(c.table.flatten().tolist())
    s = next(x for x in range(c.n_blocks) if x not in used)
    for t in (c.K, c.V, c.deg):
        t[[0, s]] = t[[s, 0]]
    c.table[c.table == 0] = s
    assert bool(c.V[0].isnan().all())


@pytest.mark.parametrize("dtype,dim,group", [("bf16", 128, 1), ("bf16", 128, 8), ("bf16", 64, 4), ("bf16", 64, 8), ("f32", 32, 2), ("f32", 64, 4),
                                             ("f32", 128, 8)])
@pytest.mark.parametrize("degrees", [True, False])
@pytest.mark.parametrize("lens", [[640, 333], [16, 5000, 700]])       # one slice and many
def test_masked_rows_that_are_no_numbers(dtype, dim, group, degrees, lens):
    print(f"masked {dtype} dim={dim} group={group} degrees={degrees} lens={lens}", flush=True)
    c = Cache(13, lens, 2, dim, 16, dtype, degrees)
    _without_block_0(c)
    for b, n in enumerate(lens):
        if n > 16:
            c.table[b, 3], c.table[b, 4], c.table[b, (n - 1) // 16] = -1, 1 << 29, -1
    if degrees:
        for b, t, d, x in ((0, 1, 0, float("nan")), (0, 15, -1, float("inf")), (1, 100, 0, float("-inf")), (1, 331, 0, float("nan"))):
            blk = int(c.table[b, t // 16])
            if t < lens[b] and blk >= 0:
                c.K[blk, :, t % 16], c.V[blk, :, t % 16], c.deg[blk, :, t % 16] = float("nan"), x, d
    q = _queries(7, len(lens), 2 * group, dim, dtype)
    K, V, deg, table, n = c.gpu()
    every = {(b, h): list(range(-(-x // 16))) for b, x in enumerate(lens) for h in range(2)}
    dense = ckv.paged_decode_attn(q.to(DEV), K, V, deg, table, n, max(lens), out_dtype=torch.float32)
    bounds, mass = ckv.paged_bounds(K, deg, table, n, max(lens))
    sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, max(lens), -(-max(lens) // 16), 16)
    sparse = ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, out_dtype=torch.float32)
    torch.cuda.synchronize()
    for o in (dense, sparse):
        assert bool(o.isfinite().all())
        _check_attention(c, q, o, every, max(lens), _scale(dim))


@pytest.mark.parametrize("dtype,dim,group", [("bf16", 128, 4), ("bf16", 64, 8), ("f32", 32, 1), ("f32", 128, 4)])
def test_an_infinite_value_of_the_last_token(dtype, dim, group):
    """Infinity in its channel, every other channel as without it: the places behind the last token count for nothing."""
    lens = [517, 33, 1, 4099]
    c = Cache(19, lens, 2, dim, 16, dtype, degrees=True)
    q = (_queries(7, len(lens), 2 * group, dim, dtype) * 0.05).to(DEV)
    K, V, deg, table, n = c.gpu()
    S = max(lens)
    flat = [torch.zeros((len(lens), 2, S) + t.shape[3:], dtype=t.dtype, device=DEV) for t in (K, V, deg)]
    for b, x in enumerate(lens):
        for f, t in zip(flat, (K, V, deg)):
            f[b, :, :x] = t[table[b, :-(-x // 16)].long()].transpose(0, 1).flatten(1, 2)[:, :x]
    P, flatP = V.clone(), flat[1].clone()
    for b, x in enumerate(lens):
        for ch, value in ((3, float("inf")), (dim - 1, float("-inf"))):
            P[int(c.table[b, (x - 1) // 16]), :, (x - 1) % 16, ch] = value
            flatP[b, :, x - 1, ch] = value
    for v0, v1, run in ((V, P, lambda v: ckv.paged_decode_attn(q, K, v, deg, table, n, S, out_dtype=torch.float32)),
                        (flat[1], flatP, lambda v: ckv.decode_attn(q, flat[0], v, lens=n, deg=flat[2], out_dtype=torch.float32))):
        plain, o = run(v0), run(v1)
        torch.cuda.synchronize()
        assert bool((o[:, :, 3] == float("inf")).all()) and bool((o[:, :, dim - 1] == float("-inf")).all())
        rest = [ch for ch in range(dim) if ch not in (3, dim - 1)]
        assert torch.equal(o[:, :, rest], plain[:, :, rest]) and bool(plain.isfinite().all())
