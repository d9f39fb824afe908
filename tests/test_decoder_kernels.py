"""What the compiler made of the kernels of cached attention and of the norm: no vector register spilled, and as many waves as their
comments count on."""
import pytest

from test_kernel_resources import _kernels


@pytest.mark.parametrize("part,count,vgprs,lds", [
    ("block_sum_kernelILi0ELi", 8, 128, 20480),          # 4 waves to a SIMD
    ("block_sum_kernelILi1ELi", 8, 128, 20480),
    ("block_sum_kernelILi2ELi", 4, 128, 16384),
    ("pair_products_kernel", 1, 64, 0),                  # 8 waves
    ("weighted_values_kernel", 1, 64, 0),
    ("ct_products_kernel", 1, 64, 0),
    ("cut_pmult_kernel", 1, 64, 0),
    ("kv_append_kernel", 1, 64, 0),
    ("conv_wide_kernelILi1E", 1, 128, 2048),             # few sources and a main prime
    ("conv_wide_kernelILi2E", 1, 128, 4096)])
def test_no_spills(part, count, vgprs, lds):
    found = {n: k for n, k in _kernels().items() if part in n}
    assert len(found) == count, sorted(found)
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
        assert k[".vgpr_count"] <= vgprs, (name, k[".vgpr_count"])
        assert k[".group_segment_fixed_size"] <= lds, (name, k[".group_segment_fixed_size"])
