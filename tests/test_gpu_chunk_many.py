"""New tokens of more than 64 sequences whose tokens are cut into parts: batches of which a few rows or all have new tokens, with lengths of none, of one part
and of several, rows of the output before the first sequence and behind the last."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_chunk import _close, _oracle, _queries, _starts
from test_gpu_chunk_parts import _is_cut
from test_gpu_sparse import DEV, Cache, _dev, _scale

pytestmark = pytest.mark.gpu

# dtype, heads, group, dim, block, sequences, of which have new tokens, longest, most new tokens, degrees, causal
CASES = [
    ("bf16", 1, 4, 64, 16, 65, 65, 3000, 3, True, True),
    ("bf16", 2, 8, 128, 16, 70, 3, 4000, 1, False, True),
    ("bf16", 2, 1, 128, 32, 200, 30, 2500, 150, True, True),
    ("bf16", 1, 4, 64, 8, 300, 300, 2000, 2, False, False),
    ("f32", 1, 2, 64, 16, 129, 100, 1500, 9, True, True),
    ("f32", 2, 4, 32, 16, 256, 5, 2000, 1, True, False),
    ("bf16", 1, 8, 128, 64, 257, 257, 700, 1, True, True),
    ("bf16", 2, 2, 64, 16, 1000, 40, 900, 10, True, True),
    ("bf16", 1, 1, 64, 16, 17000, 7, 5000, 300, False, True),    # (runs of more sequences than a wave has lanes)
]


@pytest.mark.parametrize("dtype,heads,group,dim,block,batch,active,longest,most,degrees,causal", CASES)
def test_against_the_oracle(dtype, heads, group, dim, block, batch, active, longest, most, degrees, causal):
    print(f"many {dtype} {heads}x{group} dim {dim} block {block} batch {batch} active {active} causal {causal}", flush=True)
    rng = np.random.default_rng(batch)
    lens, new = np.zeros(batch, dtype=np.int64), np.zeros(batch, dtype=np.int64)
    rows = rng.choice(batch, active, replace=False)
    new[rows] = rng.integers(1, most + 1, active)
    lens[rows] = np.maximum(rng.integers(0, longest + 1, active), new[rows])
    lens[rows[0]], lens[rows[1]] = longest, 0                    # (the second: new tokens that see nothing)
    idle = np.setdiff1d(np.arange(batch), rows)[:20]
    lens[idle] = rng.integers(0, 50, len(idle))                  # sequences that stand by
    c = Cache(107, lens.tolist(), heads, dim, block, dtype, degrees)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new, lead=5)
    q = _queries(20, starts[-1] + 4, heads * group, dim, c.dtype)
    want, bound = _oracle(c, q, new, starts, causal, _scale(dim))
    args = (q.to(DEV), K, V, deg, table, n, _dev(starts), longest)
    assert _is_cut(*args, causal=causal)
    ws = torch.full((ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), heads * group, q.shape[0], longest),), 255, dtype=torch.uint8, device=DEV)
    outs = []
    for _ in range(2):
        out = torch.full(q.shape, 7.0, dtype=c.dtype, device=DEV)
        ckv.paged_chunk_attn(*args, causal=causal, out=out, workspace=ws)
        outs.append(out)
    mine = slice(starts[0], starts[-1])
    assert (outs[0][:5] == 7.0).all() and (outs[0][starts[-1]:] == 7.0).all() and torch.equal(*outs)
    _close(outs[0][mine], want[mine], bound[mine], c.dtype)


def test_every_sequence_has_many_rows():
    """Several places a sequence, of 65 sequences, uncut: what a call of 64 of them and one of the last give."""
    lens, new = [300 + 3 * i for i in range(65)], [100 + i for i in range(65)]
    c = Cache(109, lens, 8, 64, 16)
    K, V, deg, table, n = c.gpu()
    starts = _starts(new)
    q = _queries(21, starts[-1], 8, 64, c.dtype).to(DEV)
    got = ckv.paged_chunk_attn(q, K, V, deg, table, n, _dev(starts), max(lens))
    parts = [ckv.paged_chunk_attn(q[starts[a]:starts[b]], K, V, deg, table[a:b].contiguous(), n[a:b].clone(), _dev(starts[a:b + 1]) - starts[a], max(lens))
             for a, b in ((0, 64), (64, 65))]
    want, bound = _oracle(c, q.cpu(), new, starts, True, _scale(64))
    _close(got, want, bound, c.dtype)
    for x, (a, b) in zip(parts, ((0, 64), (64, 65))):
        _close(x, want[starts[a]:starts[b]], bound[starts[a]:starts[b]], c.dtype)
