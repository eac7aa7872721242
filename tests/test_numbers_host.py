"""Numbers beyond 32 bits: the calls take int32, and what does not fit is refused instead of cut to its lower bits.  No GPU needed."""
import pytest
import torch

import paper_2506_11418_amd as ckv

BIG = 1 << 32


def _i32(*s):
    return torch.zeros(s, dtype=torch.int32)


@pytest.mark.parametrize("n", [BIG + 16, 1 << 31, -(1 << 31) - 1, 1 << 70])
def test_sizes_of_workspaces(n):
    pl = ckv.PagedLayout(2, 8, 128, ckv.BF16, 16, 100, 1000)
    for f in (lambda: ckv.paged_select_workspace(pl, n), lambda: ckv.paged_sparse_decode_attn_workspace(pl, n, 8),
              lambda: ckv.paged_sparse_decode_attn_workspace(pl, 32, n)):
        with pytest.raises(ValueError, match="32 bits"):
            f()


@pytest.mark.parametrize("n", [BIG + 16, -(BIG - 16)])
def test_numbers_of_the_calls(n):
    table, lens, free = _i32(2, 5), _i32(2), _i32(4 + 2 * 9)
    K, q = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    bounds, mass = torch.zeros(9, 2, 2, 64, dtype=torch.bfloat16), _i32(9, 2)

    def select(**kw):
        a = dict(max_len=80, n_select=2, block_size=16, n_sink=1, n_recent=1)
        a.update(kw)
        ckv.paged_select(q, bounds, mass, table, lens, **a, out=(_i32(2, 2, 2), _i32(2, 2)), workspace=torch.zeros(1 << 12, dtype=torch.uint8))
    for f in (lambda: ckv.paged_reserve(table, lens, _i32(2), free, n, 8), lambda: ckv.paged_reserve(table, lens, _i32(2), free, 16, n),
              lambda: ckv.paged_trim(table, lens, _i32(2), free, n), lambda: ckv.paged_bounds(K, None, table, lens, n, out=(bounds, mass)),
              lambda: select(max_len=n), lambda: select(n_select=n), lambda: select(block_size=n), lambda: select(n_sink=n), lambda: select(n_recent=n)):
        with pytest.raises(ValueError, match="32 bits"):
            f()


def test_rows_of_2_to_the_31_tokens():
    """A row's tokens are counted in int32: wider tables are refused, so that no length and what is added to it go beyond."""
    import ctypes as C
    p = [C.c_void_p(i << 40) for i in range(8)]           # far apart, never followed
    for width, block in ((1 << 21, 1024), (1 << 24, 128), (1 << 30, 2)):
        assert ckv.lib().ckv_paged_reserve(p[1], p[2], p[3], p[4], 1, width, 50, block, p[5], 100, p[6], p[7], None) == -2
        assert ckv.lib().ckv_paged_trim(p[1], p[2], p[3], p[4], 1, width, 50, block, None) == -2
