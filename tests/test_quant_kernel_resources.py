"""CPU tier: the quantised cache's kernels keep their state in registers (the compiler's remarks for gfx950, with the
library's own flags: no spilled vector register, no scratch memory)."""
import pytest

from tests.test_kernel_resources import test_no_spills_and_no_scratch as check


@pytest.mark.parametrize("source", ["quant.hip", "quant_decode.hip", "quant_prefill.hip"])
def test_quant_kernels(source, tmp_path):
    check(source, tmp_path)
