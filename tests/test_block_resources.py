"""Registers of a residual block's kernels, from the metadata that the compiler writes into libsoma.so: none spills, and
two blocks of a walk fit a compute unit's registers where its state leaves room."""
import pytest

from test_kernel_resources import kernels  # noqa: F401


def mine(kernels, kernel):  # noqa: F811
    return {n: k for n, k in kernels.items() if f"{len(kernel)}{kernel}" in n and "_GLOBAL__N_1" in n}


@pytest.mark.parametrize("kernel,instances", [
    ("k_la_walk", 32), ("k_la_join", 8), ("k_la_step", 4), ("k_la_share", 2), ("k_la_copy", 1), ("k_dropout", 4),
    ("k_norm_forward", 72), ("k_norm_backward", 36), ("k_norm_gain", 1), ("k_sample", 6), ("k_sample_few", 2)])
def test_no_spills(kernels, kernel, instances):  # noqa: F811
    found = mine(kernels, kernel)
    assert len(found) == instances, sorted(found)
    assert not {n for n, k in found.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}


def test_two_blocks_of_a_walk_fit_a_compute_unit(kernels):  # noqa: F811
    """Four waves a block, one on each SIMD of 512 registers."""
    walks = {n: k for n, k in mine(kernels, "k_la_walk").items() if "Li256E" not in n}
    assert walks and all(k[".vgpr_count"] <= 256 and k[".group_segment_fixed_size"] <= 80 * 1024 for k in walks.values())


def test_a_row_held_in_lds_fits_a_compute_unit(kernels):  # noqa: F811
    """What the launch adds to the kernel's own goes up to 160 KiB and no further, a rule of the host's: the kernel's own
    leaves room for the rows that it is meant for (50,257 of bf16)."""
    held = {n: k for n, k in mine(kernels, "k_sample").items() if "Li1024E" in n and "Lb1E" in n}
    assert len(held) == 2
    assert all(k[".group_segment_fixed_size"] + 2 * (50257 + 16) <= 160 * 1024 for k in held.values())
