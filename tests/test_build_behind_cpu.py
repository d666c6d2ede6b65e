"""What the compiler made of the kernels of attention behind prefixes, log probabilities, scores and eviction."""

import pytest

from tests.test_build_serving_cpu import kernels  # noqa: F401


@pytest.mark.parametrize("kernel,count", [("13prefix_kernel", 39), ("13behind_kernel", 78)])
def test_attention(kernels, kernel, count):  # noqa: F811
    """Two waves a SIMD: 256 registers a lane.  Sums and queries of the longest float32 rows do not all fit them."""
    found = {n: k for n, k in kernels.items() if kernel in n}
    assert len(found) == count
    for name, k in found.items():
        widest = "AttentionILi0ELi256ELi1ELi1E" in name or "AttentionILi0ELi256ELi1ELi2E" in name
        assert k[".vgpr_count"] <= 256, name
        assert k[".vgpr_spill_count"] <= (27 if widest else 0) and k[".private_segment_fixed_size"] <= (112 if widest else 20), name


@pytest.mark.parametrize("kernel,count,registers", [("18join_prefix_kernel", 9, 128), ("18join_behind_kernel", 78, 128), ("12score_kernel", 26, 256),
                                                    ("13select_kernel", 3, 128), ("18select_long_kernel", 1, 128), ("11move_kernel", 10, 256),
                                                    ("12sweep_kernel", 3, 128), ("13finish_kernel", 6, 128)])
def test_the_others_keep_all_in_registers(kernels, kernel, count, registers):  # noqa: F811
    found = {n: k for n, k in kernels.items() if kernel in n}
    assert len(found) == count
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
        assert k[".vgpr_count"] <= registers, name
