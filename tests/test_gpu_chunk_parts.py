"""Calls for new tokens that are cut into parts along the tokens, and the same calls uncut, where a part's numbers are the unusual ones: values
that are no finite numbers under weights that underflow, logits that are no numbers, parts in which nothing counts, scales at their limits.

A call is uncut here because rows of no sequence stand behind its own: a query tensor with more rows than the chip has places several times
over."""
import copy

import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from parity_util import f64
from test_gpu_chunk import _close, _oracle, _queries, _starts
from test_gpu_sparse import DEV, Cache, _dev

pytestmark = pytest.mark.gpu

HEADS, GROUP = 2, 8
FILL = 4 * 512 // HEADS * (128 // GROUP)     # rows of four times as many places as 256 CUs hold


def _is_cut(*args, **kw):
    """Whether a call needs a workspace for parts: it refuses one of 16 bytes."""
    try:
        ckv.paged_chunk_attn(*args, workspace=torch.empty(16, dtype=torch.uint8, device=DEV), **kw)
    except ckv.CkvError as e:
        assert e.status == -4, e
        return True
    return False


def _both(c, q, starts, scale, causal=True):
    """Outputs of the call and of the same one with rows behind that belong to no sequence: the first is cut, the second is not."""
    K, V, deg, table, n = c.gpu()
    outs = []
    for rows, cut in ((q.shape[0], True), (FILL, False)):
        dev = torch.zeros((rows, *q.shape[1:]), dtype=q.dtype, device=DEV)
        dev[:q.shape[0]] = q.to(DEV)
        args = (dev, K, V, deg, table, n, _dev(starts), max(c.lens))
        assert _is_cut(*args, scale=scale, causal=causal) == cut
        out = torch.full(dev.shape, 7.0, dtype=q.dtype, device=DEV)
        ws = torch.full((ckv.paged_chunk_attn_workspace(ckv.paged_layout_of(K, table), q.shape[1], rows, max(c.lens)),), 255, dtype=torch.uint8, device=DEV)
        ckv.paged_chunk_attn(*args, scale=scale, causal=causal, out=out, workspace=ws)
        assert (out[starts[-1]:] == 7.0).all()
        outs.append(out[:starts[-1]])
    return outs


def _token(c, b, t):
    return int(c.table[b, t // c.block]), t % c.block


@pytest.mark.parametrize("dtype,dim,causal", [("bf16", 128, True), ("bf16", 64, False), ("f32", 64, True), ("f32", 32, False)])
def test_values_that_are_no_finite_numbers_far_below_the_maximum(dtype, dim, causal):
    """Tokens 64 to 399 have logits 400 below the others': their weights underflow, in fp32 and where parts are joined.  An infinite or NaN value
    there is seen all the same."""
    print(f"far values {dtype} {dim} causal={causal}", flush=True)
    c, new = Cache(89, [1000, 700], HEADS, dim, 16, dtype), [20, 33]
    c.K[..., 0] = torch.where(c.K[..., 0].isnan(), c.K[..., 0], 0)
    for t in range(64, 400):
        blk, off = _token(c, 0, t)
        c.K[blk, :, off, 0] = -100.0
    blk, off = _token(c, 0, 200)
    c.V[blk, 0, off, 3] = float("inf")
    c.V[blk, 1, off, dim - 1] = float("nan")
    c.V[blk, 1, off, 0] = float("-inf")
    starts = _starts(new)
    q = _queries(16, starts[-1], HEADS * GROUP, dim, c.dtype)
    q[..., 0] = 8.0
    want, bound = _oracle(c, q, new, starts, causal, 0.5)
    fin = np.isfinite(want)
    hit = np.ones(fin.shape, dtype=bool)
    hit[:20, :GROUP, 3] = hit[:20, GROUP:, 0] = hit[:20, GROUP:, dim - 1] = False
    assert (fin == hit).all()
    for out, what in zip(_both(c, q, starts, 0.5, causal), ("cut", "uncut")):
        got = f64(out)
        assert (np.isfinite(got) == fin).all(), f"{what}: {np.argwhere(np.isfinite(got) != fin)[:4].tolist()}"
        _close(torch.from_numpy(np.where(fin, got, 0)), np.where(fin, want, 0), np.where(fin, bound, 0), c.dtype, what)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f32", 64)])
def test_values_that_are_no_finite_numbers_under_weights_of_zero(dtype, dim):
    """Tokens 64 to 399 have logits of -inf, in whole parts and in halves of them; an infinite value among them leaves the row none of its own."""
    print(f"values under no weight {dtype} {dim}", flush=True)
    c = Cache(103, [1000], HEADS, dim, 16, dtype)
    c.K[..., 0] = torch.where(c.K[..., 0].isnan(), c.K[..., 0], 0)
    clean = copy.deepcopy(c)
    for t in range(64, 400):
        blk, off = _token(c, 0, t)
        c.K[blk, :, off, 0] = float("-inf")
        clean.deg[blk, :, off] = 0
    for head, t, channel in ((0, 70, 1), (0, 200, 3), (1, 300, dim - 1)):
        blk, off = _token(c, 0, t)
        c.V[blk, head, off, channel] = float("inf")
    q = _queries(19, 20, HEADS * GROUP, dim, c.dtype)
    q[..., 0] = 1.0
    want, bound = _oracle(clean, q, [20], [0, 20], True, 0.5)
    fin = np.ones(want.shape, dtype=bool)
    fin[:, :GROUP, 1] = fin[:, :GROUP, 3] = fin[:, GROUP:, dim - 1] = False
    for out, what in zip(_both(c, q, [0, 20], 0.5), ("cut", "uncut")):
        got = f64(out)
        assert (np.isfinite(got) == fin).all(), f"{what}: {np.argwhere(np.isfinite(got) != fin)[:4].tolist()}"
        _close(torch.from_numpy(np.where(fin, got, 0)), np.where(fin, want, 0), np.where(fin, bound, 0), c.dtype, what)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_logits_that_are_no_numbers_in_some_parts(dtype, dim):
    """NaN keys and queries, infinite keys and queries, and stretches of several parts whose logits are all -inf or whose tokens have degree 0.  What
    the others give is compared with the oracle on a cache in which a logit of -inf is a token that does not count."""
    print(f"logits {dtype} {dim}", flush=True)
    c, new = Cache(97, [900, 1000, 640], HEADS, dim, 16, dtype), [20, 12, 70]
    c.K[..., 0] = torch.where(c.K[..., 0].isnan(), c.K[..., 0], 0)
    starts = _starts(new)
    q = _queries(17, starts[-1], HEADS * GROUP, dim, c.dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    q[starts[1]:starts[2], GROUP + 1, 0] = -0.75                 # (one head that sees the infinite keys from the other side)
    clean = copy.deepcopy(c)
    for t in range(100, 500):                                    # no weight, of whole parts
        blk, off = _token(c, 1, t)
        c.K[blk, 0, off, 0] = float("-inf")
        clean.deg[blk, 0, off] = 0
    for t in range(0, 300):
        blk, off = _token(c, 2, t)
        c.deg[blk, :, off] = clean.deg[blk, :, off] = 0
    blk, off = _token(c, 0, 300)
    c.K[blk, 0, off, 5] = float("nan")
    blk, off = _token(c, 1, 600)
    c.K[blk, 1, off, 0] = float("inf")
    clean.deg[blk, 1, off] = 0
    q[3, GROUP + 2, 7], q[5, GROUP + 3, 7] = float("nan"), float("inf")
    want, bound = _oracle(clean, torch.where(q.isfinite(), q, 0), new, starts, True, 0.25)
    nan = np.zeros(want.shape[:2], dtype=bool)
    nan[:20, :GROUP] = True
    nan[3, GROUP + 2] = nan[5, GROUP + 3] = True                 # (an infinite query meets keys of both signs)
    nan[starts[1]:starts[2], GROUP:] = True
    nan[starts[1]:starts[2], GROUP + 1] = False
    want[nan] = np.nan
    for out, what in zip(_both(c, q, starts, 0.25), ("cut", "uncut")):
        _close(out, want, bound, c.dtype, what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-6, 40.0, 1e30])
def test_scales_at_their_limits(dtype, scale):
    print(f"scale {scale} {dtype}", flush=True)
    c, new = Cache(101, [900, 513], HEADS, 64, 16, dtype), [40, 3]
    starts = _starts(new)
    q = _queries(18, starts[-1], HEADS * GROUP, 64, c.dtype)
    if scale > 100:                                              # (logits that fp32 holds)
        q = q * 1e-33
    want, bound = _oracle(c, q, new, starts, True, float(np.float32(scale)))
    for out, what in zip(_both(c, q, starts, scale), ("cut", "uncut")):
        _close(out, want, bound, c.dtype, what)
