"""What the write with strides of its own for keys and values refuses, found on the host before any launch.  No GPU needed."""
import ctypes as C

import pytest

import paper_2506_11418_amd as ckv


def _p(i, bytes=0):
    return C.c_void_p((i << 40) + bytes)        # far apart, never followed


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(slots=None), -1), (dict(n=-1), -2), (dict(kr=127), -2), (dict(kh=100), -2), (dict(vr=127), -2),
    (dict(vh=0), -2), (dict(kr=1028), -3), (dict(kh=132), -3), (dict(vr=5004), -3), (dict(vh=260), -3), (dict(v=_p(2, 8)), -3),
    # the last rows of v, and only those with v's own strides, reach into a pool
    (dict(K=_p(2, 4 * 6144 * 2 + 1024)), -1), (dict(V=_p(2, 4 * 6144 * 2 + 7 * 256)), -1), (dict(slots=None, n=0), 0)])
def test_refusals(kw, status):
    a = dict(k=_p(1), kr=1024, kh=128, v=_p(2), vr=6144, vh=128, slots=_p(3), n=5, K=_p(4), V=_p(5), deg=_p(6))
    a.update(kw)
    pl = ckv.PagedLayout(2, 8, 128, ckv.BF16, 16, 100, 1000)
    assert ckv.lib().ckv_paged_write_strided(*a.values(), C.byref(pl), None) == status
