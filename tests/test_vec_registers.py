"""Registers of the product kernels, whose speed hangs on two waves per SIMD (or blocks per CU) and on loops that touch no scratch
memory: a spill inside the large tiles' loop cost 40 % of their rate.  (What is left there is stored before the loop and loaded behind it.)"""
import pytest

from test_registers import kernels


@pytest.mark.parametrize("form,waves,scratch", [
    ("Lb1ELb1ELi2ELi4ELi8ELi4E", 2, 16),  # 256 x 256, E8M0 scales
    ("Lb1ELb1ELi2ELi2ELi4ELi4E", 2, 0),   # 128 x 128
    ("Lb0ELb1ELi2ELi2ELi4ELi4E", 2, 0),   # ... F32 scales
])
def test_product_kernels(form, waves, scratch):
    found = {k: v for k, v in kernels().items() if "k_vec_matI" in k and form in k}
    assert len(found) == 4  # pairs of factor types
    for k, (regs, bytes_) in found.items():
        assert 512 // ((regs + 7) // 8 * 8) >= waves and bytes_ <= scratch, (k, regs, bytes_)


def test_other_operators_use_no_scratch_memory():
    found = {k: v for k, v in kernels().items() if "k_vec_" in k and "k_vec_matI" not in k}
    assert len(found) > 100 and all(v[1] == 0 for v in found.values())
