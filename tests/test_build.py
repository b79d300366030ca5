"""CPU tier: what the build makes, and in which order (no compiler runs here)."""
import os
import runpy
import subprocess
import sys

import pytest


@pytest.fixture
def build_main(monkeypatch):
    """Runs the build's command line with compilers that only note their command."""
    def run(*args):
        made = []
        monkeypatch.setattr(sys, "argv", ["build", *args])
        monkeypatch.setattr(subprocess, "run",
                            lambda cmd, **_: subprocess.CompletedProcess(cmd, 0, "", ""))
        monkeypatch.setattr(os, "replace", lambda _, to: made.append(os.path.basename(to)))
        runpy.run_module("paper_2607_23815_amd.build", run_name="__main__")
        return made
    return run


def test_the_library_comes_first(build_main):
    made = build_main()
    assert made[0] == "libpkv.so" and len(made) == 2 and made[1].startswith("_tensor_address.")


def test_the_library_needs_no_torch(build_main, monkeypatch, capsys):
    """C callers and the host-only pool need hipcc alone."""
    monkeypatch.setitem(sys.modules, "torch", None)  # (an import of it raises ImportError)
    monkeypatch.delitem(sys.modules, "torch.utils.cpp_extension", raising=False)
    assert build_main() == ["libpkv.so"]
    assert "torch" in capsys.readouterr().err


def test_the_sanitized_library_alone(build_main):
    assert build_main("--sanitize") == ["libpkv_asan.so"]
