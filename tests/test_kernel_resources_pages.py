"""Registers and scratch of the kernels for new tokens over pages, from the metadata of the built library (no GPU needed)."""
from test_kernel_resources import _instances, kernels  # noqa: F401


def test_two_workgroups_of_new_tokens_share_a_cu(kernels):
    """Four waves each, one on every SIMD: 512 registers for two; a spilled sum would pass memory in every tile."""
    found = _instances(kernels, "chunk_attn_kernel")
    assert len(found) == 2 * 2 + 3 * 2             # bf16 and fp32 dims, with degrees and without
    assert all(registers <= 256 and scratch == 0 for registers, scratch in found.values()), found


def test_the_others_keep_everything_in_registers(kernels):
    names = ("chunk_merge_kernel", "chunk_merge_tail_kernel", "fork_count_kernel", "fork_deal_kernel", "compact_free_kernel", "compact_used_kernel",
             "compact_scan_kernel", "compact_blocks_kernel", "compact_rename_kernel", "compact_small_kernel", "paged_copy_kernel")
    for name in names:
        uses = [use for mangled, use in kernels.items() if mangled.startswith(f"_ZN3ckv12_GLOBAL__N_1{len(name)}{name}")]
        assert uses and all(scratch == 0 for _, scratch in uses), name
