"""The host side of the feature-map calls against a HIP runtime of the test's
own (tests/host), on the CPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host")


def run_driver(tmp_path, name, more=None):
    from paper_1706_05544_amd import build as b
    cxx = "/opt/rocm/llvm/bin/clang++"
    if not os.path.exists(cxx):
        cxx = shutil.which("clang++")
    if not cxx:
        pytest.skip("clang++ not found")
    exe = str(tmp_path / name)
    for cmd in ([cxx, "-std=c++20", "-O1", "-g", "-Wall",
                 "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                 "-I" + b.INCLUDE, "-I" + b.CSRC,
                 os.path.join(HERE, name + ".cpp")] +
                (more or [os.path.join(b.CSRC, "layers.cpp")]) +
                ["-o", exe], [exe]):
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout + r.stderr
    assert "all checks passed" in r.stdout


def test_calls_leave_the_threads_device_as_it_was(tmp_path):
    run_driver(tmp_path, "layers_device_driver")


def test_no_exception_leaves_a_call_that_finds_no_memory(tmp_path):
    # (the executable's operator new stands in for the library's)
    from paper_1706_05544_amd import native as nv
    nv.load()
    run_driver(tmp_path, "layers_memory_driver",
               [nv.LIB_PATH, "-rdynamic",
                "-Wl,-rpath," + os.path.dirname(nv.LIB_PATH)])
