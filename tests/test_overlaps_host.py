"""Buffers that a paged write, bounds, selection or sparse attention call would write over: refused on the host before any launch.
No GPU needed, and none of the calls here gets as far as a launch."""
import ctypes as C

import pytest

import paper_2506_11418_amd as ckv

EINVAL = -1


def _p(i, bytes=0):
    return C.c_void_p((i << 40) + bytes)        # far apart, never followed


def _pl(batch=2, heads=8, dim=128, dtype=ckv.BF16, bs=16, width=100, blocks=1000):
    return ckv.PagedLayout(batch, heads, dim, dtype, bs, width, blocks)


ROWS = 1000 * 8 * 16
POOL = ROWS * 128 * 2


@pytest.mark.parametrize("kw", [
    dict(deg=_p(4)), dict(deg=_p(5, POOL - 4)), dict(deg=_p(1)), dict(deg=_p(2, 5 * 2048 - 2048)), dict(deg=_p(3, 16)), dict(slots=_p(4, 64)),
    dict(slots=_p(5, POOL - 4)), dict(slots=_p(6, ROWS * 4 - 4)), dict(K=_p(2, 16)), dict(V=_p(4, POOL - 16)), dict(v=_p(5, 4096))])
def test_write(kw):
    a = dict(k=_p(1), v=_p(2), row=1024, head=128, slots=_p(3), n=5, K=_p(4), V=_p(5), deg=_p(6), pl=_pl())
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_write(*a.values(), None) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(mass=_p(1)), dict(mass=_p(2, 400)), dict(mass=_p(3)), dict(mass=_p(4, 4)), dict(mass=_p(5)), dict(mass=_p(6, 1000 * 8 * 512 - 4)),
    dict(bounds=_p(1, POOL - 16)), dict(bounds=_p(2)), dict(bounds=_p(3, 16)), dict(bounds=_p(7, 32)), dict(lens=_p(6, 4)), dict(since=_p(7, 4)),
    dict(table=_p(7, 8))])
def test_bounds(kw):
    a = dict(K=_p(1), deg=_p(2), table=_p(3), lens=_p(4), since=_p(5), pl=_pl(), n=1, bounds=_p(6), mass=_p(7))
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_bounds(*a.values(), None) == EINVAL


@pytest.mark.parametrize("out", ["sel", "sel_lens", "ws"])
@pytest.mark.parametrize("other", ["q", "bounds", "mass", "table", "lens", "sel", "sel_lens", "ws"])
def test_select(out, other):
    if out == other:
        return
    a = dict(q=_p(1), q_heads=32, bounds=_p(2), mass=_p(3), table=_p(4), lens=_p(5), pl=_pl(), max_len=1600, select=8, sink=1, recent=1,
             scale=0.0, sel=_p(6), sel_lens=_p(7), ws=_p(8), bytes=1 << 20)
    a[out] = C.c_void_p(a[other].value)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_select(*a.values(), None) == EINVAL


@pytest.mark.parametrize("out", ["o", "ws"])
@pytest.mark.parametrize("other", ["q", "K", "V", "deg", "sel", "sel_lens", "o"])
def test_sparse_attention(out, other):
    if out == other:
        return
    a = dict(q=_p(1), q_heads=32, K=_p(2), V=_p(3), deg=_p(4), sel=_p(5), sel_lens=_p(6), pl=_pl(), select=8, scale=0.0, o=_p(7), o_type=1,
             ws=_p(8), bytes=1 << 20)
    a[out] = C.c_void_p(a[other].value)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_sparse_decode_attn(*a.values(), None) == EINVAL
