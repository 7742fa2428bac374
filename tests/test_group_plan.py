"""How group norm cuts up a call (csrc/groupnorm.hpp), on the CPU: the host's
part of it compiled for this machine, with UndefinedBehaviorSanitizer."""
import math
import os
import random
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


def test_every_variant_is_compared_with_64_bits(plans):
    # of 40000 drawn calls, none takes a variant that no size of the GPU tests
    # takes (what is compiled differs between 32-bit and 16-bit types, not
    # between the two 16-bit ones)
    import test_gpu_groupnorm as a
    import test_gpu_groupnorm_variants as v

    def variants(sizes):
        cases = [s + (t, grad) for s in sizes for t in (0, 1)
                 for grad in (0, 1)]
        return {c[4:] + x: c for c, x in zip(cases, plans(cases))}

    rng = random.Random(5)
    log = lambda lo, hi: round(math.exp(rng.uniform(  # noqa: E731
        math.log(lo), math.log(hi))))
    drawn = []
    while len(drawn) < 40000:
        n, p = log(1, 200000), log(1, 100000)
        groups, each = log(1, 256), log(1, 9000)
        if rng.random() < 0.5:
            each = max(8, each // 8 * 8)
        if n * p * groups * each <= 6e7 and groups * each <= 1 << 21:
            drawn.append((n, p, groups * each, groups))
    sizes = [s for f in (a.test_group_norm_and_gradients, a.test_acts,
                         a.test_large, v.test_every_variant)
             for m in f.pytestmark
             if m.name == "parametrize" and m.args[0] == "n,p,c,groups"
             for s in m.args[1]]
    assert len(sizes) > 50
    have, reached = variants(sizes), variants(drawn)
    assert len(reached) > 120
    missing = {k: reached[k] for k in set(reached) - set(have)}
    assert not missing, missing
