"""CPU tier: bench.py's command line contract that needs no GPU -- more than one GPU is refused
with exit status 2 and a message saying why, before anything touches a device."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(*args, env=None):
    return subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), *args], cwd=ROOT,
                          capture_output=True, text=True, timeout=300, env=env)


def test_more_than_one_gpu_is_refused():
    r = _run("--gpus", "2")
    assert r.returncode == 2
    assert "one GPU" in r.stderr and r.stdout == ""


def test_a_multi_rank_launch_is_refused():
    env = dict(os.environ, WORLD_SIZE="4")
    r = _run(env=env)
    assert r.returncode == 2
    assert "one GPU" in r.stderr and r.stdout == ""


def test_the_committed_traffic_is_of_these_kernels():
    """The bytes that the benchmark reports come from counters of the kernels' present sources: files
    that several kernels share do not change for one that is not among them."""
    import bench
    for kernel in bench.KERNEL_SOURCES:
        assert bench.traffic_from_profiles(kernel), kernel
