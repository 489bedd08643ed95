"""Registers of the first-order operators' kernels, from the metadata that the compiler writes into libsoma.so: none
spills, since a spill's loads and stores would stand in the queue of the tiles that are on their way."""
import pytest

from test_kernel_resources import kernels  # noqa: F401


@pytest.mark.parametrize("kernel,instances", [
    ("k_ce_mm", 16), ("k_ce_rows", 5), ("k_ce_pack", 2), ("k_ce_max", 2), ("k_ce_sum", 4), ("k_ce_join", 2), ("k_scan_forward", 3),
    ("k_scan_forward_maps", 3), ("k_scan_backward", 3), ("k_scan_backward_maps", 3), ("k_scan_step", 2), ("k_adamw", 2),
    ("k_adamw_moments", 1)])
def test_no_spills(kernels, kernel, instances):  # noqa: F811
    mine = {n: k for n, k in kernels.items() if f"{len(kernel)}{kernel}" in n and "_GLOBAL__N_1" in n}
    assert len(mine) == instances, sorted(mine)
    assert not {n for n, k in mine.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}


def test_two_blocks_of_a_scan_fit_a_compute_unit(kernels):  # noqa: F811
    """Blocks of 8 waves, two on each SIMD of 512 registers: 128 a lane leave room for another block."""
    mine = {n: k[".vgpr_count"] for n, k in kernels.items() if "k_scan_forward" in n or "k_scan_backward" in n}
    assert mine and all(v <= 128 for v in mine.values()), mine
