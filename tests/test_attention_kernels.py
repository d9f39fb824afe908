"""What the compiler made of the attention kernels and of the key-switch variants they use: nothing spilled, and as many waves as their
comments count on."""
import pytest

from test_kernel_resources import _kernels


def _named(part):
    return {n: k for n, k in _kernels().items() if part in n}


@pytest.mark.parametrize("part,count,vgprs", [
    ("rot_sum_kernelILi0E", 2, 72),                      # 7 waves to a SIMD, 8
    ("rot_sum_kernelILi1E", 2, 64),
    ("rot_sum_kernelILi2E", 2, 64),
    ("prod_sum_kernelILb1E", 5, 96),
    ("prod_sum_kernelILb0E", 5, 168),
    ("inner_c_kernelILi16ELi1E", 1, 168),                # weighted and mapped: 3 waves, as the plain one
    ("inner_c_kernelILi16ELi2E", 1, 168),
    ("inner8_kernelILi2ELb1ELi1E", 1, 168),
    ("inner8_kernelILi2ELb1ELi2E", 1, 168),
    ("inner8_kernelILi1ELb0ELi1E", 1, 168)])
def test_no_spills(part, count, vgprs):
    found = _named(part)
    assert len(found) == count, sorted(found)
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
        assert k[".vgpr_count"] <= vgprs, (name, k[".vgpr_count"])
