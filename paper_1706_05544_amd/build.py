"""Build libmi355svm.so (HIP for gfx950) in-tree with hipcc.

Usage: python -m paper_1706_05544_amd.build
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmi355svm.so")

ARCH = "gfx950"
DEVICE_SOURCES = ["kernels.hip", "rows.hip", "lockstep.hip", "select.hip",
                  "predict.hip", "noalloc.hip", "iterate.hip", "factor.hip",
                  "resident.hip", "linear.hip", "matmul.hip", "norm.hip", "hinge.hip",
                  "adamw.hip", "gradnorm.hip", "linear4.hip",
                  "groupnorm.hip", "groupgrad.hip"]
HOST_SOURCES = ["solver.cpp", "api.cpp", "layers.cpp", "network.cpp",
                "steps.cpp"]

# Packed fp32 instructions are disabled for every compilation that has a
# device pass (hipcc runs one for the .cpp sources too).
COMMON = ["-O3", "-fPIC", "-std=c++20", "-Wall", "-Wno-unused-result",
          "--offload-arch=" + ARCH, "-Xclang", "-target-feature", "-Xclang",
          "-packed-fp32-ops", "-I" + INCLUDE]
DEVICE_FLAGS = ["-x", "hip", "-munsafe-fp-atomics"]
# roctx ranges of the host phases (rocprofv3 --marker-trace)
LINK = ["-L/opt/rocm/lib", "-lrocprofiler-sdk-roctx", "-Wl,-rpath,/opt/rocm/lib"]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc",
              shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src: str, device: bool, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [_hipcc()] + COMMON + (DEVICE_FLAGS if device else []) + [
        "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("compile failed: %s\n%s%s" % (src, r.stdout,
                                                         r.stderr))
    if verbose and r.stderr.strip():
        print(r.stderr, file=sys.stderr)
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source for gfx950 and link the shared library."""
    os.makedirs(BUILD, exist_ok=True)
    jobs = [(s, True) for s in DEVICE_SOURCES] + [(s, False)
                                                  for s in HOST_SOURCES]
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(lambda j: _compile(j[0], j[1], verbose), jobs))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [_hipcc(), "-shared", "-fPIC", "--offload-arch=" + ARCH, "-o", tmp
           ] + objs + LINK
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
