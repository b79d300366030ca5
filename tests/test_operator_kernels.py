"""CPU tier: the kernels around sparse reads keep their state in registers, as the other kernels do
(tests/test_kernel_resources.py): no spilled vector register and no scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2607_23815_amd import build as b
from tests.test_kernel_resources import test_no_spills_and_no_scratch as _check


@pytest.mark.parametrize("source", ["select.hip", "sparse.hip", "rope.hip"])
def test_no_spills_and_no_scratch(source, tmp_path):
    _check(source, tmp_path)


@pytest.mark.parametrize("source,kernels", [("bounds.hip", 4), ("tables.hip", 3)])
def test_no_spills_and_no_scratch_in_small_files(source, kernels, tmp_path):
    """(The other files' check expects more kernels of a file than these hold.)"""
    try:
        hipcc = b.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not found")
    r = subprocess.run([hipcc, "-O3"] + b.FLAGS +
                       ["--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                        os.path.join(b.CSRC, source), "-o", str(tmp_path / "out.o")],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    names, spills, scratch = (re.findall(p, r.stderr) for p in (
        r"Function Name: (\S+)", r"VGPRs Spill: (\d+)", r"ScratchSize \[bytes/lane\]: (\d+)"))
    assert len(names) == len(spills) == len(scratch) == kernels, r.stderr[-2000:]
    assert not [x for x in zip(names, spills, scratch) if x[1] != "0" or x[2] != "0"]
