"""The native binding makes the calls of a paged step itself (0, not None), with arguments in the library's order; and buffers that lie
next to one another in one allocation are no overlap."""
import numpy as np
import pytest
import torch

import paper_2506_11418_amd as ckv
from test_gpu_sparse import DEV, Cache, _check_attention, _dev, _queries
from test_gpu_write_strides import _Never, _Recorder

pytestmark = pytest.mark.gpu


class _Arena:
    """Tensors one behind the other, without a gap where their alignment needs none."""

    def __init__(self, bytes):
        self.memory, self.at = torch.zeros(bytes, dtype=torch.uint8, device=DEV), 0

    def take(self, t, align=16):
        self.at = -(-self.at // align) * align
        n = t.numel() * t.element_size()
        out = self.memory[self.at:self.at + n].view(t.dtype).view(t.shape)
        self.at += n
        out.copy_(t)
        return out


@pytest.mark.parametrize("dtype,degrees,since", [("bf16", True, True), ("f32", False, False)])
def test_the_binding_makes_every_call(monkeypatch, dtype, degrees, since):
    block, heads, dim, n_select, batch = 16, 4, 64, 6, 3
    outs = []
    native = _Recorder(ckv._binding())
    for module in (native, _Never()):
        monkeypatch.setattr(ckv, "_native", module)
        c = Cache(17, [300, 5, 161], heads, dim, block, dtype, degrees, spare=20, room=4)
        K, V, deg, table, lens = c.gpu()
        free = ckv.paged_free_list(c.n_blocks)
        used = sorted(set(table[table >= 0].tolist()))
        left = [x for x in range(c.n_blocks) if x not in used]
        free[0] = len(left)
        free[4:4 + len(left)] = _dev(left)
        free[4 + c.n_blocks:][torch.tensor(used, device=DEV)] = 2**31 - 1
        a, i32 = _Arena(1 << 25), lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        before = lens.clone()
        slots = ckv.paged_reserve(table, lens, _dev([1, 9, 2]), free, block, 14, out=tuple(a.take(i32(n), 4) for n in (14, batch + 1, batch)))[0]
        ckv.paged_trim(table, lens, _dev([-1, 13, -1]), free, block)
        g = torch.Generator().manual_seed(1)
        k, v = (a.take(torch.randn(14, heads, dim, generator=g).to(c.dtype).to(DEV)) for _ in range(2))
        ckv.paged_write(k, v, slots, K, V, deg)
        q = a.take(_queries(3, batch, heads * 2, dim, dtype).to(DEV))
        b = (a.take(torch.zeros(c.n_blocks, heads, 2, dim, dtype=c.dtype, device=DEV)), a.take(i32(c.n_blocks, heads), 4))
        ckv.paged_bounds(K, deg, table, lens, 400, out=b)
        if since:
            ckv.paged_bounds(K, deg, table, lens, 9, since=before, out=b)
        pl = ckv.paged_layout_of(K, table)
        out = (a.take(i32(batch, heads, n_select), 4), a.take(i32(batch, heads), 4))
        ws = a.take(torch.zeros(ckv.paged_select_workspace(pl, 400), dtype=torch.uint8, device=DEV))
        ckv.paged_select(q, *b, table, lens, 400, n_select, block, n_sink=2, n_recent=1, scale=0.25, out=out, workspace=ws)
        ws = a.take(torch.zeros(ckv.paged_sparse_decode_attn_workspace(pl, heads * 2, n_select), dtype=torch.uint8, device=DEV))
        o = a.take(torch.zeros(q.shape, dtype=torch.float32, device=DEV))
        ckv.paged_sparse_decode_attn(q, K, V, deg, *out, scale=0.25, out=o, workspace=ws)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (slots, table, lens, free, K, V, *b, *out, o)])
        c.K, c.V, c.deg, c.table, c.lens = K.cpu(), V.cpu(), c.deg if deg is None else deg.cpu(), table.cpu(), lens.tolist()
        if deg is None:
            c.deg[:] = 1
        want, tokens, picked = c.want_select(q.cpu(), b[0].cpu(), b[1].cpu(), 400, n_select, 2, 1, 0.25)
        assert np.array_equal(out[0].cpu().numpy(), want) and np.array_equal(out[1].cpu().numpy(), tokens)
        _check_attention(c, q.cpu(), o, picked, 400, 0.25)
    names = ["paged_reserve", "paged_trim", "paged_write", "paged_bounds"] + ["paged_bounds"] * since + ["paged_select", "paged_sparse_decode_attn"]
    assert native.took == [(n, 0) for n in names]
    for x, y in zip(*outs):
        assert torch.equal(x.nan_to_num(), y.nan_to_num()) if x.is_floating_point() else torch.equal(x, y)
