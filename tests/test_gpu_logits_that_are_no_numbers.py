"""Decode attention where a logit is no number: the softmax of that query head is NaN, and so is its output, not zero.  The other heads
are as without it."""
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_sparse import DEV, DT

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 128, 4, 40), ("bf16", 64, 8, 5000), ("bf16", 128, 8, 33000), ("f32", 64, 2, 70), ("f32", 128, 4, 3000), ("f32", 128, 8, 40000)]


def _caches(dtype, dim, L, seed):
    """(K, V) strided [1, 2, L, dim], the same on pages of 16 with a table, and lens."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    K, V = (torch.randn(1, 2, L, dim, generator=g, device=DEV).to(DT[dtype]) for _ in range(2))
    nb = -(-L // 16)
    table = torch.randperm(nb + 3, generator=g, device=DEV)[:nb].to(torch.int32).view(1, nb)

    def pages(x):
        pool = torch.full((nb + 3, 2, 16, dim), float("nan"), dtype=x.dtype, device=DEV)
        rows = torch.full((2, nb * 16, dim), float("nan"), dtype=x.dtype, device=DEV)
        rows[:, :L] = x[0]
        pool[table[0].long()] = rows.view(2, nb, 16, dim).transpose(0, 1)
        return pool
    return K, V, pages, table, torch.tensor([L], dtype=torch.int32, device=DEV)


def _runs(q, K, V, pages, table, lens, out_dtype):
    Kp, Vp, L = pages(K), pages(V), K.shape[2]
    yield "strided", ckv.decode_attn(q, K, V, out_dtype=out_dtype)
    yield "paged", ckv.paged_decode_attn(q, Kp, Vp, None, table, lens, L, out_dtype=out_dtype)
    bounds, mass = ckv.paged_bounds(Kp, None, table, lens, L)
    sel, sel_lens = ckv.paged_select(q, bounds, mass, table, lens, L, table.shape[1], 16)
    yield "sparse", ckv.paged_sparse_decode_attn(q, Kp, Vp, None, sel, sel_lens, out_dtype=out_dtype)


@pytest.mark.parametrize("dtype,dim,group,L", SHAPES)
@pytest.mark.parametrize("what", ["query nan", "query inf", "key nan", "key inf"])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_nan_logits(dtype, dim, group, L, what, out_dtype):
    print(f"nan logits {dtype} dim={dim} group={group} L={L} {what}", flush=True)
    K, V, pages, table, lens = _caches(dtype, dim, L, L + group)
    q = torch.randn(1, 2 * group, dim, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(DT[dtype])
    q[0, :group, 3] = q[0, :group, 3].abs() + 0.5        # (an infinite key is an infinite logit of every head)
    plain = dict(_runs(q, K, V, pages, table, lens, out_dtype))
    bad = list(range(group)) if what.startswith("key") else [group - 1]
    x = float(what.split()[1])
    if what.startswith("key"):
        K[0, 0, L // 3, 3] = x
    else:
        q[0, group - 1, 3] = x
    for name, o in _runs(q, K, V, pages, table, lens, out_dtype):
        torch.cuda.synchronize()
        assert bool(o[0, bad].isnan().all()), name
        rest = [h for h in range(2 * group) if h not in bad]
        # (the reference that weights refer to moves at other tokens when a head of the group does not ask for it: a rounding of the weights
        # and of their sums, 2^-16 of the largest value in all, and one of each output)
        step = 2.0**-16 * V.float().abs().max() + (2.0**-7 if out_dtype == torch.bfloat16 else 0.0) * plain[name][0, rest].float().abs()
        assert bool(((o[0, rest].float() - plain[name][0, rest].float()).abs() <= step).all()), name


def test_an_empty_cache_is_still_zero():
    K, V, pages, table, lens = _caches("bf16", 64, 40, 3)
    q = torch.full((1, 8, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    lens.zero_()
    assert not ckv.decode_attn(q, K, V, lens=lens).any() and not ckv.paged_decode_attn(q, pages(K), pages(V), None, table, lens, 40).any()
