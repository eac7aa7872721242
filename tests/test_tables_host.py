"""What the table, slot and selection calls refuse, found on the host before any launch; and their sizes.  No GPU needed."""
import ctypes as C
import re
import struct

import pytest
import torch

import paper_2506_11418_amd as ckv

Z = None


def _p(i):
    return C.c_void_p(i << 40)        # far apart, never followed


def _reserve(**kw):
    a = dict(table=_p(1), lens=_p(2), new=_p(3), free=_p(4), batch=3, width=10, blocks=50, bs=16, slots=_p(5), n=100, starts=_p(6), ok=_p(7))
    a.update(kw)
    return ckv.lib().ckv_paged_reserve(*a.values(), Z)


@pytest.mark.parametrize("kw,status", [
    (dict(table=Z), -1), (dict(lens=Z), -1), (dict(new=Z), -1), (dict(free=Z), -1), (dict(slots=Z), -1),
    (dict(batch=0), -2), (dict(batch=4097), -2), (dict(width=0), -2), (dict(blocks=0), -2), (dict(bs=24), -2), (dict(bs=2048), -2),
    (dict(n=-1), -2), (dict(n=(1 << 30) + 1), -2), (dict(batch=4096, width=1 << 19, bs=1), -2),
    (dict(blocks=1 << 27, bs=16), -5), (dict(table=C.c_void_p((1 << 40) + 2)), -3), (dict(slots=C.c_void_p((5 << 40) + 1)), -3),
    (dict(new=_p(2)), -1), (dict(slots=_p(1)), -1), (dict(starts=C.c_void_p((4 << 40) + 64)), -1), (dict(ok=_p(6)), -1),
])
def test_reserve_refuses(kw, status):
    assert _reserve(**kw) == status


@pytest.mark.parametrize("args,status", [
    ((Z, _p(2), _p(3), _p(4), 3, 10, 50, 16), -1), ((_p(1), Z, _p(3), _p(4), 3, 10, 50, 16), -1),
    ((_p(1), _p(2), Z, _p(4), 3, 10, 50, 16), -1), ((_p(1), _p(2), _p(3), Z, 3, 10, 50, 16), -1),
    ((_p(1), _p(2), _p(2), _p(4), 3, 10, 50, 16), -1), ((_p(1), _p(2), _p(3), _p(1), 3, 10, 50, 16), -1),
    ((_p(1), _p(2), _p(3), _p(4), 5000, 10, 50, 16), -2),
    ((_p(1), _p(2), _p(3), _p(4), 3, 10, 50, 3), -2), ((_p(1), C.c_void_p((2 << 40) + 2), _p(3), _p(4), 3, 10, 50, 16), -3),
])
def test_trim_refuses(args, status):
    assert ckv.lib().ckv_paged_trim(*args, Z) == status


def test_free_refuses():
    f = ckv.lib().ckv_paged_free
    assert f(Z, 3, _p(1), 10, Z) == -1 and f(_p(2), 3, Z, 10, Z) == -1 and f(_p(2), -1, _p(1), 10, Z) == -2
    assert f(_p(2), 3, _p(1), 0, Z) == -2 and f(_p(1), 3, _p(1), 10, Z) == -1 and f(C.c_void_p((2 << 40) + 1), 3, _p(1), 10, Z) == -3


def _pl(batch=2, heads=8, dim=128, dtype=ckv.BF16, bs=16, width=100, blocks=1000):
    return ckv.PagedLayout(batch, heads, dim, dtype, bs, width, blocks)


@pytest.mark.parametrize("kw,status", [
    (dict(k=Z), -1), (dict(v=Z), -1), (dict(slots=Z), -1), (dict(K=Z), -1), (dict(V=Z), -1), (dict(n=-1), -2),
    (dict(row=127), -2), (dict(head=100), -2), (dict(row=1028), -3), (dict(head=132), -3), (dict(k=C.c_void_p((1 << 40) + 8)), -3),
    (dict(k=_p(4)), -1), (dict(V=_p(4)), -1), (dict(pl=_pl(blocks=1 << 28)), -5), (dict(pl=_pl(dim=100)), -3), (dict(pl=_pl(bs=12)), -2),
])
def test_write_refuses(kw, status):
    a = dict(k=_p(1), v=_p(2), row=1024, head=128, slots=_p(3), n=5, K=_p(4), V=_p(5), deg=_p(6), pl=_pl())
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_write(*a.values(), Z) == status


@pytest.mark.parametrize("kw,status", [
    (dict(K=Z), -1), (dict(table=Z), -1), (dict(lens=Z), -1), (dict(bounds=Z), -1), (dict(mass=Z), -1), (dict(n=0), -2), (dict(n=-3), -2),
    (dict(bounds=_p(1)), -1), (dict(pl=_pl(dim=32)), -5), (dict(pl=_pl(dim=256)), -5), (dict(pl=_pl(blocks=1 << 24)), -5),
    (dict(bounds=C.c_void_p((6 << 40) + 8)), -3), (dict(since=C.c_void_p((5 << 40) + 2)), -3),
])
def test_bounds_refuses(kw, status):
    a = dict(K=_p(1), deg=_p(2), table=_p(3), lens=_p(4), since=_p(5), pl=_pl(), n=1, bounds=_p(6), mass=_p(7))
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_bounds(*a.values(), Z) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=Z), -1), (dict(bounds=Z), -1), (dict(mass=Z), -1), (dict(table=Z), -1), (dict(lens=Z), -1), (dict(sel=Z), -1),
    (dict(sel_lens=Z), -1), (dict(ws=Z), -1), (dict(q_heads=31), -2), (dict(q_heads=24), -5), (dict(q_heads=128), -5), (dict(max_len=0), -2),
    (dict(select=0), -2), (dict(select=1 << 28), -2), (dict(sink=-1), -1), (dict(sink=5, recent=4), -1), (dict(recent=-2), -1),
    (dict(bytes=256), -4), (dict(pl=_pl(dim=32)), -5), (dict(q=C.c_void_p((1 << 40) + 8)), -3), (dict(sel=C.c_void_p((6 << 40) + 2)), -3),
])
def test_select_refuses(kw, status):
    a = dict(q=_p(1), q_heads=32, bounds=_p(2), mass=_p(3), table=_p(4), lens=_p(5), pl=_pl(), max_len=1600, select=8, sink=1, recent=1,
             scale=0.0, sel=_p(6), sel_lens=_p(7), ws=_p(8), bytes=1 << 20)
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_select(*a.values(), Z) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=Z), -1), (dict(K=Z), -1), (dict(sel=Z), -1), (dict(sel_lens=Z), -1), (dict(o=Z), -1), (dict(ws=Z), -1), (dict(q_heads=12), -2),
    (dict(q_heads=24), -5), (dict(select=0), -2), (dict(select=1 << 28), -2), (dict(bytes=0), -4), (dict(o_type=5), -1),
    (dict(pl=_pl(batch=10000)), -5), (dict(pl=_pl(dim=32)), -5), (dict(K=C.c_void_p((2 << 40) + 4)), -3),
])
def test_sparse_attention_refuses(kw, status):
    a = dict(q=_p(1), q_heads=32, K=_p(2), V=_p(3), deg=_p(4), sel=_p(5), sel_lens=_p(6), pl=_pl(), select=8, scale=0.0, o=_p(7), o_type=1,
             ws=_p(8), bytes=1 << 20)
    a.update(kw)
    a["pl"] = C.byref(a["pl"])
    assert ckv.lib().ckv_paged_sparse_decode_attn(*a.values(), Z) == status


@pytest.mark.parametrize("pl", [_pl(), _pl(batch=1, heads=1), _pl(bs=64, width=7), _pl(dtype=ckv.F32, dim=32, batch=60)])
def test_workspaces_serve_shorter_lengths(pl):
    sizes = [ckv.paged_select_workspace(pl, n) for n in (1, 15, 16, 17, 500, 1600, 1 << 20)]
    assert sizes == sorted(sizes)
    assert sizes[-1] >= 4 * pl.batch * pl.heads * pl.max_blocks
    for n_select in (1, 7, 256):
        assert ckv.paged_sparse_decode_attn_workspace(pl, pl.heads * 4, n_select) >= 4 * pl.batch * pl.heads


def test_python_refuses_what_does_not_fit_together():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    table, lens, free = i32(2, 5), i32(2), i32(4 + 2 * 9)
    with pytest.raises(ValueError, match="current GPU"):             # tensors of the host
        ckv.paged_reserve(table, lens, i32(2), free, 16, 8)
    with pytest.raises(ValueError, match="current GPU"):
        ckv.paged_trim(table, lens, i32(2), free, 16)
    for bad in (dict(lens=i32(3)), dict(lens=lens.long()), dict(free=i32(5)), dict(free=i32(23)), dict(table=i32(5, 2).t()), dict(n=-1),
                dict(out=(i32(7), i32(3), i32(2))), dict(out=(i32(8), i32(2), i32(2)))):
        a = dict(table=table, lens=lens, new=i32(2), free=free, bs=16, n=8, out=None)
        a.update(bad)
        with pytest.raises(ValueError):
            ckv.paged_reserve(*a.values())
    K = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for bad in (dict(k=k.float()), dict(k=k[:3]), dict(V=K.float()), dict(k=torch.zeros(4, 3, 64, dtype=torch.bfloat16)[:, :2]), dict(slots=i32(4).long()),
                dict(deg=i32(9, 2, 8)), dict(K=K.transpose(0, 1)), dict()):
        a = dict(k=k, v=k, slots=i32(4), K=K, V=K, deg=None)
        a.update(bad)
        with pytest.raises(ValueError):
            ckv.paged_write(*a.values())
    q, bounds, mass = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(9, 2, 2, 64, dtype=torch.bfloat16), i32(9, 2)
    for bad in (dict(q=q[:1]), dict(bounds=bounds.float()), dict(bounds=bounds[:8]), dict(mass=i32(9, 2).t()), dict(lens=i32(1)), dict(select=0), dict()):
        a = dict(q=q, bounds=bounds, mass=mass, table=table, lens=lens, max_len=80, select=2, bs=16)
        a.update(bad)
        with pytest.raises((ValueError, RuntimeError)):              # (without a GPU torch has no output to give either)
            ckv.paged_select(*a.values(), out=(i32(2, 2, max(a["select"], 1)), i32(2, 2)), workspace=torch.zeros(1 << 12, dtype=torch.uint8))
    for bad in (dict(q=q.float()), dict(sel=i32(2, 3, 2)), dict(sel_lens=i32(4)), dict(out=q.half()), dict(out=q[:, :4]), dict()):
        a = dict(q=q, K=K, V=K, deg=None, sel=i32(2, 2, 2), sel_lens=i32(2, 2), scale=0.0, out_dtype=None, out=torch.zeros_like(q),
                 ws=torch.zeros(1 << 16, dtype=torch.uint8))
        a.update(bad)
        with pytest.raises(ValueError):
            ckv.paged_sparse_decode_attn(*a.values())
    with pytest.raises(ValueError):
        ckv.paged_bounds(K, None, table, lens, 80, out=(bounds, mass))
    with pytest.raises(ValueError):
        ckv.paged_free(i32(3).long(), free)
    with pytest.raises(ValueError):
        ckv.paged_free_list(0)


class _OnGpu(torch.Tensor):
    """A host tensor that says it lives on the GPU; nothing here follows its pointer."""
    is_cuda = property(lambda self: True)
    get_device = lambda self: 0


def _made_calls():
    t = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype).as_subclass(_OnGpu)
    h = lambda *s: t(*s, dtype=torch.bfloat16)
    table, lens, free, ws = t(2, 4), t(2), t(4 + 2 * 6), t(1 << 16, dtype=torch.uint8)
    pool, bounds, mass, q, sel, sel_lens = h(6, 2, 16, 64), h(6, 2, 2, 64), t(6, 2), h(2, 8, 64), t(2, 2, 3), t(2, 2)
    return {
        "ckv_paged_reserve": lambda: ckv.paged_reserve(table, lens, t(2), free, 16, 5, out=(t(5), t(3), t(2))),
        "ckv_paged_trim": lambda: ckv.paged_trim(table, lens, t(2), free, 16),
        "ckv_paged_write": lambda: ckv.paged_write(h(5, 2, 64), h(5, 2, 64), t(5), pool, pool, t(6, 2, 16)),
        "ckv_paged_bounds": lambda: ckv.paged_bounds(pool, None, table, lens, 9, out=(bounds, mass)),
        "ckv_paged_select": lambda: ckv.paged_select(q, bounds, mass, table, lens, 64, 3, 16, out=(sel, sel_lens), workspace=ws),
        "ckv_paged_sparse_decode_attn": lambda: ckv.paged_sparse_decode_attn(q, pool, pool, None, sel, sel_lens, out=q, workspace=ws),
    }


@pytest.mark.parametrize("name", list(_made_calls()))
@pytest.mark.parametrize("status", [-6, -2, None])
def test_a_call_is_made_once_by_either_route(monkeypatch, name, status):
    """A status of the binding ends the call; None goes on to ctypes, which makes it once."""
    class Answer:
        def __getattr__(self, _):
            return lambda *a: status

    class Calls:
        made, real = [], ckv.lib()

        def __getattr__(self, n):
            if n == "ckv_strerror":
                return self.real.ckv_strerror
            return lambda *a: self.made.append(n) or 0
    calls = Calls()
    Calls.made = []
    monkeypatch.setattr(ckv, "lib", lambda: calls)
    monkeypatch.setattr(ckv, "_here", lambda: (0, 0))
    monkeypatch.setattr(ckv, "_stream", lambda: None)
    monkeypatch.setattr(ckv, "_native", Answer())
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    if status is None:
        _made_calls()[name]()
        assert Calls.made == [name]
    else:
        with pytest.raises(ckv.CkvError) as e:
            _made_calls()[name]()
        assert e.value.status == status and str(e.value).startswith(name + ":") and not Calls.made


def test_registers_of_the_paged_kernels():
    """No scratch, and the waves a SIMD that the launches count on."""
    pytest.importorskip("msgpack")
    from test_kernel_resources import LIB, _instances, _metadata
    data, found = open(LIB, "rb").read(), {}
    for at in (m.start() for m in re.finditer(b"\x7fELF", data)):
        if struct.unpack_from("<H", data, at + 18)[0] == 224:       # EM_AMDGPU
            found.update({k[".name"]: (k[".vgpr_count"], k[".private_segment_fixed_size"]) for k in _metadata(data[at:])})
    mine = {k: v for k, v in found.items() if re.search("N_1[0-9]+paged_(score|select|bounds|reserve|return|write)_kernel", k)}
    assert len(mine) > 30 and all(scratch == 0 for _, scratch in mine.values())
    scores = _instances(found, "paged_score_kernel")
    assert len(scores) == 5 * 4 and all(use[0] <= 168 for k, use in scores.items() if k[0] == "DF16b" and (k[1], k[2]) != ("128", "8"))
