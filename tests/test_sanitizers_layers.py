"""The feature-map calls' host code (argument checks, workspace layouts)
under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: the build
of test_sanitizers.py with a driver of its own
(tests/sanitize/layers_driver.c)."""
import os
import shutil

import pytest

import test_sanitizers as ts


def test_layers_validation_under_asan_ubsan(tmp_path):
    from paper_1706_05544_amd import build as b
    llvm = "/opt/rocm/llvm/bin"
    if not os.path.exists(os.path.join(llvm, "clang++")) or \
            not shutil.which("gcc"):
        pytest.skip("ROCm clang not found")
    host_san = []
    for f in ts.SAN[:3]:
        host_san += ["-Xarch_host", f]
    objs = []
    for src in b.HOST_SOURCES:
        o = str(tmp_path / (src + ".o"))
        ts._run([b._hipcc()] + [c for c in b.COMMON if c != "-O3"] +
                ["-O1", "-g"] + host_san +
                ["-c", os.path.join(b.CSRC, src), "-o", o])
        objs.append(o)
    drv = str(tmp_path / "driver.o")
    ts._run([os.path.join(llvm, "clang"), "-std=c11"] + ts.SAN +
            ["-I" + b.INCLUDE, "-c", os.path.join(ts.HERE, "layers_driver.c"),
             "-o", drv])
    exe = str(tmp_path / "layers_asan")
    ts._run([os.path.join(llvm, "clang++")] + ts.SAN[:1] +
            ["-o", exe, drv] + objs + ts._device_objects() +
            ["-L/opt/rocm/lib", "-lamdhip64"] + b.LINK)
    r = ts._run([exe], env=ts.ENV, timeout=300)
    assert "all checks passed" in r.stdout
