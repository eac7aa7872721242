"""What the calls for new tokens over pages, forks, compaction and copies refuse, found on the host before any launch; and their sizes.
No GPU needed."""
import ctypes as C

import pytest
import torch

import paper_2506_11418_amd as ckv

Z = None


def _p(i, bytes=0):
    return C.c_void_p((i << 42) + bytes)        # far apart, never followed


def _pl(batch=2, heads=8, dim=128, dtype=ckv.BF16, bs=16, width=100, blocks=1000):
    return ckv.PagedLayout(batch, heads, dim, dtype, bs, width, blocks)


POOL = 1000 * 8 * 16 * 128 * 2


def _chunk(**kw):
    a = dict(q=_p(1), row=6144, head=128, q_heads=32, starts=_p(2), n=20, K=_p(3), V=_p(4), deg=_p(5), table=_p(6), lens=_p(7), pl=_pl(), max_len=1600,
             scale=0.0, causal=1, o=_p(8), o_type=1, ws=_p(9), bytes=1 << 30)
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    return ckv.lib().ckv_paged_chunk_attn(*a.values(), Z)


@pytest.mark.parametrize("kw,status", [
    (dict(q=Z), -1), (dict(starts=Z), -1), (dict(K=Z), -1), (dict(V=Z), -1), (dict(table=Z), -1), (dict(lens=Z), -1), (dict(o=Z), -1), (dict(ws=Z), -1),
    (dict(o_type=2), -1), (dict(n=-1), -2), (dict(max_len=0), -2), (dict(q_heads=0), -2), (dict(q_heads=30), -2), (dict(row=127), -2), (dict(head=64), -2),
    (dict(row=0), -2), (dict(q_heads=24), -5), (dict(q_heads=128), -5), (dict(pl=_pl(dim=96)), -5), (dict(pl=_pl(dim=32)), -5), (dict(pl=_pl(dim=256)), -5),
    (dict(pl=_pl(dim=16, dtype=ckv.F32)), -5), (dict(pl=_pl(blocks=1 << 24)), -5), (dict(pl=_pl(bs=12)), -2), (dict(pl=_pl(batch=0)), -2),
    (dict(row=6148), -3), (dict(head=132), -3), (dict(q=_p(1, 8)), -3), (dict(o=_p(8, 8)), -3), (dict(ws=_p(9, 4)), -3), (dict(starts=_p(2, 2)), -3),
    (dict(bytes=0), -4), (dict(bytes=1000), -4), (dict(scale=1e-31), -5), (dict(scale=2e30), -5), (dict(scale=float("inf")), -5),
    (dict(o=_p(1, 4096)), -1), (dict(o=_p(3, POOL - 16)), -1), (dict(o=_p(4)), -1), (dict(o=_p(5)), -1), (dict(o=_p(6, 16)), -1), (dict(o=_p(9)), -1),
    (dict(ws=_p(1)), -1), (dict(ws=_p(3, 64)), -1), (dict(ws=_p(7)), -1), (dict(ws=_p(2)), -1), (dict(lens=_p(8, 32)), -1), (dict(starts=_p(8)), -1),
    (dict(pl=_pl(batch=65536)), -5), (dict(pl=_pl(batch=1, bs=1, width=(1 << 31) - 1000), max_len=(1 << 31) - 1), -5),
    (dict(pl=_pl(batch=1, bs=1, width=(1 << 31) - 1000), max_len=(1 << 31) - 1024), -5), (dict(n=(1 << 30) + 1), -5), (dict(n=1 << 30), -5),
    (dict(scale=float("-inf"), q=Z), -1), (dict(scale=1e-30, o=_p(1)), -1), (dict(scale=1e30, o=_p(1)), -1),
])
def test_chunk_attention_refuses(kw, status):
    assert _chunk(**kw) == status


def test_chunk_attention_of_no_tokens():
    assert _chunk(n=0, q=Z, starts=Z, o=Z, ws=Z, bytes=0) == 0


@pytest.mark.parametrize("heads,q_heads,dim", [(8, 32, 128), (1, 1, 64), (2, 16, 128), (40, 40, 64)])
def test_a_workspace_serves_smaller_calls(heads, q_heads, dim):
    """The size for n tokens and max_len is enough for fewer and shorter ones, of any batch: such calls get past the check of the workspace,
    to the one for overlaps."""
    size = lambda n, m, b: ckv.paged_chunk_attn_workspace(_pl(batch=b, heads=heads, dim=dim), q_heads, n, m)
    last = 0
    for n in (0, 1, 2, 3, 7, 16, 31, 32, 33, 64, 100, 255, 512, 1000, 1024, 2000, 4096, 5000, 100000):
        row = [size(n, m, 3) for m in (1, 100, 256, 257, 1000, 5000, 16384, 1 << 20)]
        assert row == sorted(row) and row[-1] >= last and row == [size(n, m, 999) for m in (1, 100, 256, 257, 1000, 5000, 16384, 1 << 20)]
        last = row[-1]
        for b in (1, 2, 5, 64, 1000):
            for m in (1, 257, 5000, 1 << 20):
                want = size(n, m, b)
                a = dict(pl=_pl(batch=b, heads=heads, dim=dim, width=1 << 17, blocks=100), q_heads=q_heads, n=n, max_len=m, row=q_heads * dim, head=dim)
                # (an output over the queries: refused as an overlap, after the workspace was found large enough)
                assert n == 0 or _chunk(**a, bytes=want, o=_p(1)) == -1, (n, m, b)
    assert last < 1 << 28


def test_numbers_beyond_32_bits():
    big = (1 << 32) + 16
    pl = _pl()
    for f in (lambda: ckv.paged_chunk_attn_workspace(pl, big, 5, 5), lambda: ckv.paged_chunk_attn_workspace(pl, 32, big, 5),
              lambda: ckv.paged_chunk_attn_workspace(pl, 32, 5, big), lambda: ckv.paged_compact_workspace(big)):
        with pytest.raises(ValueError, match="32 bits"):
            f()
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    K = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    for f in (lambda: ckv.paged_chunk_attn(q, K, K.clone(), None, i(2, 5), i(2), i(3), big), lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(22), big, 4),
              lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(22), 16, big), lambda: ckv.paged_compact(i(2, 5), i(2), i(22), 16, big),
              lambda: ckv.paged_compact(i(2, 5), i(2), i(22), big, 3)):
        with pytest.raises(ValueError, match="32 bits"):
            f()


@pytest.mark.parametrize("kw", [
    dict(q=torch.zeros(3, 8, 64)), dict(q=torch.zeros(3, 8, 128, dtype=torch.bfloat16)), dict(q=torch.zeros(24, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3, 64, 8, dtype=torch.bfloat16).transpose(1, 2)), dict(lens=torch.zeros(3, dtype=torch.int32)),
    dict(lens=torch.zeros(2, dtype=torch.int64)), dict(starts=torch.zeros(2, dtype=torch.int32)), dict(table=torch.zeros(2, 5)),
    dict(deg=torch.zeros(9, 2, 8, dtype=torch.int32)), dict(V=torch.zeros(9, 2, 16, 64)), dict(out=torch.zeros(3, 8, 64, dtype=torch.float16)),
    dict(out=torch.zeros(3, 4, 64)), dict()])
def test_chunk_attention_refuses_tensors(kw):
    """(The last one: nothing is wrong but that the tensors are not on a GPU.)"""
    K = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)
    a = dict(q=torch.zeros(3, 8, 64, dtype=torch.bfloat16), K=K, V=K.clone(), deg=None, table=torch.zeros(2, 5, dtype=torch.int32),
             lens=torch.zeros(2, dtype=torch.int32), starts=torch.zeros(3, dtype=torch.int32), max_len=80)
    out = kw.pop("out", None)
    a.update(kw)
    with pytest.raises(ValueError):
        ckv.paged_chunk_attn(*a.values(), out=out)


def _fork(**kw):
    a = dict(table=_p(1), lens=_p(2), source=_p(3), free=_p(4), batch=3, width=10, blocks=50, bs=16, moves=_p(5), n=100, granted=_p(6))
    a.update(kw)
    return ckv.lib().ckv_paged_fork(*a.values(), Z)


@pytest.mark.parametrize("kw,status", [
    (dict(table=Z), -1), (dict(lens=Z), -1), (dict(source=Z), -1), (dict(free=Z), -1), (dict(moves=Z), -1), (dict(granted=Z), -1),
    (dict(batch=0), -2), (dict(batch=4097), -2), (dict(width=0), -2), (dict(blocks=0), -2), (dict(bs=24), -2), (dict(n=-1), -2), (dict(n=(1 << 30) + 1), -2),
    (dict(blocks=1 << 27), -5), (dict(table=_p(1, 2)), -3), (dict(moves=_p(5, 1)), -3), (dict(granted=_p(6, 2)), -3),
    (dict(source=_p(2)), -1), (dict(moves=_p(1, 8)), -1), (dict(granted=_p(5, 796)), -1), (dict(granted=_p(4, 64)), -1), (dict(source=_p(6)), -1),
])
def test_fork_refuses(kw, status):
    assert _fork(**kw) == status


def _compact(**kw):
    a = dict(table=_p(1), lens=_p(2), free=_p(3), batch=3, width=10, blocks=50, bs=16, moves=_p(4), n=100, extent=_p(5), ws=_p(6), bytes=4096)
    a.update(kw)
    return ckv.lib().ckv_paged_compact(*a.values(), Z)


@pytest.mark.parametrize("kw,status", [
    (dict(table=Z), -1), (dict(lens=Z), -1), (dict(free=Z), -1), (dict(moves=Z), -1), (dict(extent=Z), -1), (dict(ws=Z), -1),
    (dict(batch=0), -2), (dict(batch=4097), -2), (dict(blocks=0), -2), (dict(bs=3), -2), (dict(n=-1), -2), (dict(blocks=1 << 27), -5),
    (dict(ws=_p(6, 8)), -3), (dict(extent=_p(5, 2)), -3), (dict(bytes=64), -4), (dict(bytes=0), -4),
    (dict(extent=_p(2, 8)), -1), (dict(moves=_p(1, 116)), -1), (dict(ws=_p(3, 16)), -1), (dict(extent=_p(6, 64)), -1), (dict(lens=_p(1)), -1),
])
def test_compact_refuses(kw, status):
    assert _compact(**kw) == status


def test_compact_workspace():
    for n in (1, 31, 32, 33, 1000, 1 << 20):
        words = -(-n // 32)                  # a byte and four bits a block, and what is counted
        assert 64 + 48 * words <= ckv.paged_compact_workspace(n) < 64 + 48 * words + 256
        assert _compact(blocks=n, bytes=ckv.paged_compact_workspace(n), extent=_p(2)) == -1      # (large enough: the overlap is found next)
    for n in (0, -5):
        with pytest.raises(ckv.CkvError):
            ckv.paged_compact_workspace(n)


@pytest.mark.parametrize("kw,status", [
    (dict(moves=Z), -1), (dict(K=Z), -1), (dict(V=Z), -1), (dict(bounds=Z), -1), (dict(mass=Z), -1), (dict(n=-1), -2), (dict(n=(1 << 30) + 1), -2),
    (dict(n=1 << 30), -5), (dict(n=2796202, moves=_p(3, 64)), -1), (dict(n=2796203, moves=_p(3, 64)), -5),
    (dict(pl=_pl(dim=100)), -3), (dict(pl=_pl(bs=12)), -2), (dict(pl=_pl(heads=1 << 14, dim=1 << 8)), -2),
    (dict(K=_p(2, 8)), -3), (dict(bounds=_p(5, 4)), -3), (dict(moves=_p(1, 2)), -3), (dict(mass=_p(6, 1)), -3),
    (dict(V=_p(2, POOL - 16)), -1), (dict(moves=_p(3, 64)), -1), (dict(deg=_p(2)), -1), (dict(bounds=_p(4, 16)), -1), (dict(mass=_p(1, 8)), -1),
])
def test_copy_refuses(kw, status):
    a = dict(moves=_p(1), n=5, K=_p(2), V=_p(3), deg=_p(4), bounds=_p(5), mass=_p(6), pl=_pl())
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_copy(*a.values(), Z) == status


def test_pages_refuse_tensors():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    K = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)
    bad = [lambda: ckv.paged_fork(i(2, 5), i(2), i(3), i(22), 16, 4), lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(21), 16, 4),
           lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(22), 16, -1), lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(22), 16, 4, out=(i(3, 2), i(2))),
           lambda: ckv.paged_fork(i(2, 5), i(2), i(2), i(22), 16, 4, out=(i(4, 2), i(3))), lambda: ckv.paged_compact(i(2, 5), i(3), i(22), 16, 4),
           lambda: ckv.paged_compact(i(2, 5), i(2), i(22), 16, -2), lambda: ckv.paged_compact(i(2, 5), i(2), i(22), 16, 4, out=(i(4, 2), i(2))),
           lambda: ckv.paged_copy(i(4), K, K.clone()), lambda: ckv.paged_copy(i(4, 3), K, K.clone()), lambda: ckv.paged_copy(i(4, 2).long(), K, K.clone()),
           lambda: ckv.paged_copy(i(4, 2), K, K.float()), lambda: ckv.paged_copy(i(4, 2), K, K.clone(), None, torch.zeros(9, 2, 2, 64, dtype=torch.bfloat16)),
           lambda: ckv.paged_copy(i(4, 2), K, K.clone(), None, torch.zeros(9, 2, 2, 32, dtype=torch.bfloat16), i(9, 2)),
           lambda: ckv.paged_copy(i(4, 2), K, K.clone(), i(9, 2, 8))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
