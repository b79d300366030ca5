"""CPU tier: the kernels around sparse reads keep their state in registers, as the other kernels do
(tests/test_kernel_resources.py): no spilled vector register and no scratch memory."""
import pytest

from tests.test_kernel_resources import test_no_spills_and_no_scratch as _check


@pytest.mark.parametrize("source", ["select.hip", "sparse.hip", "rope.hip"])
def test_no_spills_and_no_scratch(source, tmp_path):
    _check(source, tmp_path)
