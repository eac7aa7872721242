"""The selection at its edges: scores of zero of either sign, NaN keys of either sign, and rows so long that the last step takes
several spans."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from parity_util import i64
from test_gpu_sparse import DEV, Cache, _queries, _same, _scale

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_round_to_zero_of_either_sign_are_equal(dtype):
    """Products below the smallest fp32 number: every score is zero, and ties go to the lower block."""
    c = Cache(14, [24, 9], 1, 64, 1, dtype, degrees=False)
    for b, n in enumerate(c.lens):
        sign = torch.where(torch.arange(n) % 3 == 0, -1.0, 1.0).to(c.dtype)
        c.K[c.table[b, :n].long()] = (torch.ones(n, 1, 1, 64, dtype=c.dtype) * 1e-30) * sign[:, None, None, None]
    q = torch.full((2, 2, 64), 1e-30).to(c.dtype)
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 24)
    sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, 24, 5, 1, n_sink=0, n_recent=0)
    torch.cuda.synchronize()
    want, tokens, picked = c.want_select(q, bounds.cpu(), mass.cpu(), 24, 5, 0, 0, _scale(64))
    assert picked[0, 0] == list(range(5))
    assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), tokens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_of_nan_keys_of_either_sign(dtype):
    """Both bounds of the channel are NaN, whichever sign the key's NaN has."""
    c = Cache(8, [40, 33], 2, 64, 16, dtype)
    blk, other = int(c.table[0, 0]), int(c.table[1, 2])
    bits = c.K.view(torch.int16 if dtype == "bf16" else torch.int32)
    quiet, odd = (0x7fc0, 0x7f81) if dtype == "bf16" else (0x7fc00000, 0x7f800001)       # (quiet, and as close to infinity as there is)
    least = -2**15 if dtype == "bf16" else -2**31
    bits[blk, 0, 3, 5], bits[blk, 0, 4, 6], bits[blk, 1, 0, 0], bits[blk, 1, 15, 63] = quiet, least + quiet, least + odd, odd
    bits[other, 1, 0, 9] = least + quiet     # (the block's only token)
    assert int(c.K.isnan()[blk].sum()) == 4
    K, _, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, 40)
    torch.cuda.synchronize()
    wb, wm = c.want_bounds(torch.zeros(bounds.shape, dtype=c.dtype), torch.zeros(mass.shape, dtype=torch.int32))
    for b, h, ch in ((blk, 0, 5), (blk, 0, 6), (blk, 1, 0), (blk, 1, 63), (other, 1, 9)):
        wb[b, h, :, ch] = float("nan")
    assert _same(bounds, wb) and torch.equal(mass.cpu(), wm)


@pytest.mark.parametrize("few", [False, True])         # few: three different keys, so that the cut falls among equal ones
def test_a_last_step_of_several_spans(few):
    """More than 32 segments of a row that keep 512 keys each: 35 * 512 keys in the last step, which takes 16384 at a time."""
    tokens, n_select = 70000, 514
    c = Cache(16, [tokens, 40000], 1, 32, 1, "f32", degrees=False)
    q = _queries(10, 2, 2, 32, "f32")
    if few:
        q = q.abs()
        value = torch.ones(tokens)
        value[::200] = 2.0
        value[-2500:-1800:4] = 3.0           # (175 of these are taken, and the others among the 350 before)
        for b, n in enumerate(c.lens):
            c.K[c.table[b, :n].long(), 0, 0] = value[:n, None].expand(n, 32)
    K, V, deg, table, n = c.gpu()
    bounds, mass = ckv.paged_bounds(K, deg, table, n, tokens)
    for n_sink, n_recent in ((1, 1), (0, 2)):
        sel, sel_lens = ckv.paged_select(q.to(DEV), bounds, mass, table, n, tokens, n_select, 1, n_sink, n_recent)
        torch.cuda.synchronize()
        want, count, picked = c.want_select(q, bounds.cpu(), mass.cpu(), tokens, n_select, n_sink, n_recent, _scale(32))
        if few:                              # the cut lies among equal keys of the last step's second span
            twos = [i for i in picked[0, 0] if value[i] == 2.0]
            assert twos[0] < 32 * 2048 < twos[-1] < max(i for i in range(tokens) if value[i] == 2.0)
        assert np.array_equal(i64(sel), want) and np.array_equal(i64(sel_lens), count), (n_sink, n_recent)
