"""Argument checks of the calls around a feature network's step and its
serving: every refusal comes before any device call, so these run without a
GPU (the pointers are never followed)."""
import ctypes as ct
import os
import subprocess

import pytest

from paper_1706_05544_amd import native as nv

INV, UNS = nv.SVM_E_INVALID, nv.SVM_E_UNSUPPORTED
needs_no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"),
                                  reason="a GPU is present")


def ref(a):
    return None if a is None else ct.byref(a)


# ---------------------------------------------------- norm and clipped step


def grad_norm(n=300, count=1, scale=1.0, most=1.0, norm=1 << 20,
              factor=1 << 21, work=1 << 22, nbytes=1 << 30, device=0,
              null=False, **fields):
    g = nv.svm_grad(1 << 23, n, 0)
    for k, v in fields.items():
        setattr(g, k, v)
    return nv.load().svm_grad_norm(
        None if null else ct.addressof(g), count, scale, most, norm, factor,
        work, nbytes, device, None)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(null=True), dict(n=-1), dict(n=1 << 41),
    dict(dtype=3), dict(dtype=-1), dict(data=None), dict(data=(1 << 23) + 2),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(most=-1.0),
    dict(most=float("nan")), dict(norm=None), dict(norm=(1 << 20) + 2),
    dict(factor=(1 << 21) + 1), dict(factor=1 << 20), dict(work=None),
    dict(work=(1 << 22) + 8), dict(nbytes=7), dict(device=-1)])
def test_grad_norm_refusals(kw):
    assert grad_norm(**kw) == INV
    assert nv.svm_last_error()


@needs_no_gpu
def test_grad_norm_accepted():
    for kw in (dict(), dict(factor=None), dict(most=float("inf")),
               dict(n=0, data=None, work=None, nbytes=0),
               dict(count=0, null=True, work=None), dict(scale=-2.0)):
        assert grad_norm(**kw) == nv.SVM_E_DEVICE


def test_grad_norm_workspace():
    lib, n = nv.load(), ct.c_int64(-1)
    g = nv.svm_grad(1 << 23, 100000, 1)
    assert lib.svm_grad_norm_workspace(ct.addressof(g), 1, None) == INV
    assert lib.svm_grad_norm_workspace(None, 1, ct.byref(n)) == INV
    assert lib.svm_grad_norm_workspace(ct.addressof(g), 1, ct.byref(n)) == 0
    assert n.value >= 8
    # the longest there may be: no more than some sums for each launch
    g.n = 1 << 40
    assert lib.svm_grad_norm_workspace(ct.addressof(g), 1, ct.byref(n)) == 0
    assert 8 <= n.value <= 1 << 23


def clipped(factor=16, n=300, null=False, **fields):
    t = nv.svm_adamw_tensor(16, 32, None, 64, 80, None, None, n, 0, 0)
    for k, v in fields.items():
        setattr(t, k, v)
    p = nv.svm_adamw_params(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 1, 32)
    return nv.load().svm_adamw_step_clipped(
        ct.addressof(t), 1, None if null else ct.byref(p), factor, 0, None)


@pytest.mark.parametrize("kw", [
    dict(factor=18), dict(null=True), dict(n=-1), dict(param=None),
    dict(m=72), dict(dtype=5)])
def test_clipped_step_refusals(kw):
    assert clipped(**kw) == INV
    assert nv.svm_last_error()


@needs_no_gpu
def test_clipped_step_accepted():
    assert clipped() == nv.SVM_E_DEVICE
    assert clipped(factor=None) == nv.SVM_E_DEVICE


# ------------------------------------------------------------------ structs


def layout(tmp_path, what):
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n'
                    '#include "mi355svm.h"\nint main(void) {\n%s'
                    '  return 0;\n}\n' % "".join(
                        '  printf("%%zu ", %s);\n' % w for w in what))
    inc = os.path.join(os.path.dirname(os.path.dirname(
        os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-std=c99", "-I", inc, str(prog), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True,
                         check=True).stdout
    return [int(x) for x in out.split()]


def test_gradient_layout_matches_header(tmp_path):
    got = layout(tmp_path, ["sizeof(svm_grad)", "offsetof(svm_grad, n)",
                            "offsetof(svm_grad, dtype)"])
    assert got == [ct.sizeof(nv.svm_grad), nv.svm_grad.n.offset,
                   nv.svm_grad.dtype.offset]
    # the table that the binding fills column by column is the same struct
    r = nv._GRAD_ROW
    assert r.itemsize == ct.sizeof(nv.svm_grad)
    for name, _ in nv.svm_grad._fields_:
        assert r.fields[name][1] == getattr(nv.svm_grad, name).offset
