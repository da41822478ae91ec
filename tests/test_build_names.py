"""The kernels that the build looks at for scratch memory are those that there are: every name stands for a compiled kernel, and the
products of 8-bit integers are looked at in both their forms."""
import pytest

from paper_2309_14717_amd import build as b
from test_build_guard import REMARK

TILES = "_ZN6qalora14gemm_i8_kernelILb0ELi256ELi256ELi2ELi4ELi2ELb0EEEvNS_12Int8GemmArgsE"
MIXED = "_ZN6qalora20gemm_i8_mixed_kernelILb0ELi192EEEvNS_12Int8GemmArgsEi"


@pytest.mark.parametrize("name", [TILES, MIXED])
def test_products_of_8_bit_integers_may_not_spill(name):
    b._check_no_scratch("gemm_i8.hip", REMARK.format(name=name, scratch=0))
    with pytest.raises(RuntimeError, match="scratch"):
        b._check_no_scratch("gemm_i8.hip", REMARK.format(name=name, scratch=16))


def test_a_name_without_a_kernel_is_refused():
    both = REMARK.format(name=TILES, scratch=0) + REMARK.format(name=MIXED, scratch=0)
    b._check_names("gemm_i8.hip", both)
    for one in (TILES, MIXED):
        with pytest.raises(RuntimeError, match="no kernel"):
            b._check_names("gemm_i8.hip", REMARK.format(name=one, scratch=0))
