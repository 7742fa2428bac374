"""How group norm cuts up a call (csrc/groupnorm.hpp), on the CPU: the host's
part of it compiled for this machine, with UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

from paper_1706_05544_amd import build as b

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """f(cases) -> the variant of each case (samples, positions, channels,
    groups, type, gradient): (threads, pieces, even, chunks)."""
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    san = ["-fsanitize=undefined", "-fno-sanitize-recover=all"]
    cmd = [b._hipcc(), "-std=c++20", "-O1", "-x", "hip",
           "--offload-host-only", "-I" + b.INCLUDE, "-I" + b.CSRC]
    for f in san:
        cmd += ["-Xarch_host", f]
    r = subprocess.run(cmd + [os.path.join(HERE, "group_plan_driver.cpp"),
                              "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(cases):
        text = "".join("%d %d %d %d %d %d\n" % tuple(c) for c in cases)
        r = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        out = [tuple(map(int, x.split())) for x in r.stdout.splitlines()]
        assert len(out) == len(cases)
        return out

    return ask


def test_no_samples_of_any_number_of_positions(plans):
    for positions in (1, 2 ** 31 - 1, 2 ** 40, 2 ** 62, 2 ** 63 - 1):
        for channels, groups in ((64, 8), (1, 1), (1 << 21, 1), (231, 33)):
            for t in range(3):
                plans([(0, positions, channels, groups, t, grad)
                       for grad in (0, 1)])


def test_the_kernels_assumptions_hold_for_every_plan(plans):
    # (the driver checks each)
    sizes = [1, 2, 3, 5, 8, 9, 16, 31, 49, 64, 100, 196, 500, 1024, 3977,
             8192, 70001]
    cases = []
    for n in (1, 2, 5, 33, 300, 4096, 100000):
        for p in sizes:
            for c, groups in ((1, 1), (7, 7), (8, 1), (24, 3), (30, 3), (64, 8),
                              (231, 33), (256, 8), (504, 7), (640, 32),
                              (1000, 4), (1000, 1000), (4096, 1), (4098, 2),
                              (5000, 1), (9000, 2), (16384, 4), (1 << 21, 1),
                              (1 << 21, 1 << 21)):
                cases += [(n, p, c, groups, t, grad) for t in range(3)
                          for grad in (0, 1)]
    plans(cases)
