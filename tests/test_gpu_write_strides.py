"""Ragged rows whose keys and values lie differently in memory, by either route, against indexing."""
import pytest
import torch

import paper_2506_11418_amd as ckv

pytestmark = pytest.mark.gpu
DEV = "cuda"


class _Recorder:
    """The native binding, with what its calls returned."""

    def __init__(self, real):
        self.real, self.took = real, []

    def __getattr__(self, name):
        def call(*a):
            self.took.append((name, getattr(self.real, name)(*a)))
            return self.took[-1][1]
        return call


class _Never:
    def __getattr__(self, name):
        return lambda *a: None


def _rows(kind, n, heads, dim, dt, g):
    x = torch.randn(n, 3 * heads + 2, dim, generator=g).to(dt).to(DEV)
    if kind == "plain":
        return x[:, :heads].contiguous()
    if kind == "fused":
        return x[:, heads:2 * heads]
    if kind == "heads_first":
        return x[:, :heads].transpose(0, 1).contiguous().transpose(0, 1)
    return x.view(n, -1)[:, dim:(heads + 1) * dim].unflatten(1, (heads, dim))          # "flat": of a row of one projection


@pytest.mark.parametrize("k_kind,v_kind", [("plain", "fused"), ("fused", "plain"), ("heads_first", "flat"), ("flat", "heads_first"), ("fused", "fused")])
@pytest.mark.parametrize("dtype,heads,dim,block,n", [("bf16", 8, 128, 16, 64), ("bf16", 8, 128, 16, 2001), ("bf16", 2, 64, 32, 1), ("bf16", 1, 64, 8, 77),
                                                     ("bf16", 1, 128, 16, 1), ("f32", 3, 36, 4, 500), ("f32", 1, 4, 2, 9)])
def test_keys_and_values_with_strides_of_their_own(monkeypatch, k_kind, v_kind, dtype, heads, dim, block, n):
    print(f"write {k_kind}/{v_kind} {dtype} heads={heads} dim={dim} n={n}", flush=True)
    dt, g = torch.bfloat16 if dtype == "bf16" else torch.float32, torch.Generator().manual_seed(n + heads)
    k, v = _rows(k_kind, n, heads, dim, dt, g), _rows(v_kind, n, heads, dim, dt, g)
    assert k.shape == v.shape == (n, heads, dim)
    n_blocks = n // block + 3
    slots = torch.randperm(n_blocks * block, generator=g)[:n].to(torch.int32)
    if n > 5:
        slots[3] = -1
    K, V = (torch.randn(n_blocks, heads, block, dim, generator=g).to(dt) for _ in range(2))
    deg = torch.full((n_blocks, heads, block), 7, dtype=torch.int32)
    wK, wV, wd, s = K.clone(), V.clone(), deg.clone(), slots.long()
    at = s >= 0
    wK[s[at] // block, :, s[at] % block], wV[s[at] // block, :, s[at] % block], wd[s[at] // block, :, s[at] % block] = k.cpu()[at], v.cpu()[at], 1
    native = _Recorder(ckv._binding())
    for module in (native, _Never()):
        monkeypatch.setattr(ckv, "_native", module)
        Kd, Vd, dd = K.to(DEV), V.to(DEV), deg.to(DEV)
        ckv.paged_write(k, v, slots.to(DEV), Kd, Vd, dd)
        torch.cuda.synchronize()
        assert torch.equal(Kd.cpu(), wK) and torch.equal(Vd.cpu(), wV) and torch.equal(dd.cpu(), wd)
    assert native.took == [("paged_write", 0)]
