"""Block selection for queries that are no numbers: no block of their KV head has a finite score."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from parity_util import i64
from test_gpu_sparse import DEV, Cache, _check_attention, _queries, _scale

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,group", [("bf16", 1), ("bf16", 4), ("bf16", 8), ("f32", 2), ("f32", 4), ("f32", 8)])
@pytest.mark.parametrize("bad", [float("nan"), float("-inf")])
def test_a_query_that_is_no_number_ranks_its_blocks_in_order(dtype, group, bad):
    """No block of its KV head has a finite score, whatever the group's other heads say; the other KV head selects by its scores."""
    print(f"query {bad} {dtype} group={group}", flush=True)
    c = Cache(13, [16 * 40, 16 * 40], 2, 64, 16, dtype)
    q = _queries(7, 2, 2 * group, 64, dtype)
    q[0, group - 1, 3] = q[1, 2 * group - 1, 63] = bad
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 640)
    for n_select in (3, 11, 38):
        sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, 640, n_select, 16, n_sink=0, n_recent=1)
        torch.cuda.synchronize()
        want, tokens, picked = c.want_select(q, bounds.cpu(), mass.cpu(), 640, n_select, 0, 1, _scale(64))
        assert picked[0, 0][:-1] == picked[1, 1][:-1] == list(range(n_select - 1)) and picked[0, 1] != picked[0, 0]
        assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), tokens), n_select
    # the group's other heads attend to those blocks as with a query of numbers
    o = ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, out_dtype=torch.float32)
    q[0, group - 1, 3] = q[1, 2 * group - 1, 63] = 0.0
    plain = ckv.paged_sparse_decode_attn(q.to(DEV), K, V, deg, sel, sel_lens, out_dtype=torch.float32)
    torch.cuda.synchronize()
    o[0, group - 1], o[1, 2 * group - 1] = plain[0, group - 1], plain[1, 2 * group - 1]
    _check_attention(c, q, o, picked, 640, _scale(64))
