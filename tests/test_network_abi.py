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


# -------------------------------------------------------- weights in 4 bits


def arr(rows, cols, at=1 << 20, ld=None, dtype=nv.SVM_F32, dev=1):
    return nv.svm_array(at, rows, cols, cols if ld is None else ld, dtype,
                        dev)


def packed(rows=40, cols=100, at=1 << 28, nbytes=1 << 20, group=32,
           dtype=nv.SVM_F32):
    return nv.svm_packed(at, nbytes, rows, cols, group, dtype)


BAD_PACKED = [packed(rows=0), packed(cols=0), packed(rows=(1 << 21) + 1),
              packed(cols=(1 << 21) + 1), packed(group=16), packed(group=96),
              packed(group=0), packed(dtype=3), packed(dtype=-1),
              packed(at=None), packed(at=(1 << 28) + 8),
              # 3 tiles of 16 x 128: 1024 bytes of codes each, 4 * 48 scales
              packed(nbytes=3 * 1024 + 4 * 48 * 4 - 1), packed(nbytes=-1)]


def test_pack4_bytes():
    lib, n = nv.load(), ct.c_int64(-1)
    for args, want in (((40, 100, 32, 0), 3 * 1024 + 4 * 48 * 4),
                       ((40, 100, 128, 1), 3 * 1024 + 48 * 2),
                       ((1, 1, 64, 2), 1024 + 2 * 16 * 2),
                       ((1 << 21, 1 << 21, 128, 0), (1 << 41) + (1 << 37))):
        assert lib.svm_pack_weights_bytes(*args, ct.byref(n)) == 0
        assert n.value == want
    for args in ((0, 1, 32, 0), (1, 0, 32, 0), (1, 1, 33, 0), (1, 1, 32, 3),
                 ((1 << 21) + 1, 1, 32, 0)):
        assert lib.svm_pack_weights_bytes(*args, ct.byref(n)) == INV
        assert n.value == 0
    assert lib.svm_pack_weights_bytes(1, 1, 32, 0, None) == INV


def pack(W=None, P=None, device=0, fn="svm_pack_weights"):
    W, P = W or arr(40, 100), P or packed()
    if fn == "svm_pack_weights":
        return nv.load().svm_pack_weights(ref(W), ref(P), device, None)
    return nv.load().svm_unpack_weights(ref(P), ref(W), device, None)


@pytest.mark.parametrize("fn", ["svm_pack_weights", "svm_unpack_weights"])
def test_pack4_refusals(fn):
    for P in BAD_PACKED:
        assert pack(P=P, fn=fn) == INV
        assert nv.svm_last_error()
    for W in (arr(40, 99), arr(39, 100), arr(40, 100, dtype=1),
              arr(40, 100, ld=99), arr(40, 100, at=None),
              arr(40, 100, at=(1 << 20) + 2), arr(40, 100, at=1 << 28),
              arr(40, 100, at=(1 << 28) + 3 * 1024)):
        assert pack(W=W, fn=fn) == INV
    assert pack(W=arr(40, 100, dev=0), fn=fn) == UNS
    assert pack(device=-1, fn=fn) == INV
    lib = nv.load()
    assert lib.svm_pack_weights(None, ref(packed()), 0, None) == INV
    assert lib.svm_pack_weights(ref(arr(40, 100)), None, 0, None) == INV
    assert lib.svm_unpack_weights(None, ref(arr(40, 100)), 0, None) == INV
    assert lib.svm_unpack_weights(ref(packed()), None, 0, None) == INV


def linear4(X=None, P=None, b=None, R=None, act=0, Y=None, work=16,
            nbytes=1 << 40, device=0):
    X, P = X or arr(6, 100), P or packed()
    Y = Y or arr(X.rows, 40, at=3 << 20)
    return nv.load().svm_linear_packed(ref(X), ref(P), ref(b), ref(R), act,
                                       ref(Y), work, nbytes, device, None)


@pytest.mark.parametrize("kw", [dict(P=P) for P in BAD_PACKED] + [
    dict(act=6), dict(act=-1), dict(X=arr(6, 99)), dict(X=arr(-1, 100)),
    dict(X=arr(6, 100, dtype=1)), dict(X=arr(6, 100, at=None)),
    dict(b=arr(1, 39, at=4 << 20)), dict(b=arr(40, 1, at=4 << 20)),
    dict(R=arr(6, 39, at=4 << 20)), dict(Y=arr(6, 39, at=3 << 20)),
    dict(Y=arr(5, 40, at=3 << 20)), dict(Y=arr(6, 40)),
    dict(Y=arr(6, 40, at=1 << 28)), dict(R=arr(6, 40, at=(3 << 20) + 16)),
    dict(R=arr(6, 40, at=3 << 20, ld=41)), dict(device=-1), dict(work=17),
    # many rows need the unpacked weights
    dict(X=arr(5000, 100, at=5 << 28), Y=arr(5000, 40, at=6 << 28),
         work=None)])
def test_linear4_refusals(kw):
    assert linear4(**kw) == INV
    assert nv.svm_last_error()


@needs_no_gpu
def test_packed_weights_accepted():
    assert pack() == nv.SVM_E_DEVICE
    assert pack(fn="svm_unpack_weights") == nv.SVM_E_DEVICE
    assert linear4() == nv.SVM_E_DEVICE
    assert linear4(R=arr(6, 40, at=3 << 20)) == nv.SVM_E_DEVICE  # in place
    assert linear4(X=arr(0, 100, at=None), work=None) == nv.SVM_E_DEVICE
    assert linear4(P=packed(nbytes=3 * 1024 + 4 * 48 * 4)) == nv.SVM_E_DEVICE


def test_packed4_layout_matches_header(tmp_path):
    S = nv.svm_packed
    names = [n for n, _ in S._fields_]
    got = layout(tmp_path, ["sizeof(svm_packed)"] + [
        "offsetof(svm_packed, %s)" % n for n in names])
    assert got == [ct.sizeof(S)] + [getattr(S, n).offset for n in names]


# --------------------------------------------------------------- group norm


def group(X=None, positions=3, groups=2, w=None, b=None, eps=1e-5, act=0,
          Y=None, mean=None, rstd=None, work=16, nbytes=1 << 40, device=0):
    X, Y = X or arr(6, 4), Y or arr(6, 4, at=2 << 20)
    return nv.load().svm_group_norm(
        ref(X), positions, groups, ref(w), ref(b), eps, act, ref(Y), mean,
        rstd, work, nbytes, device, None)


GROUPS = [dict(positions=0), dict(positions=-3), dict(positions=4),
          dict(positions=7), dict(groups=0), dict(groups=-1), dict(groups=3),
          dict(groups=5)]


@pytest.mark.parametrize("kw", GROUPS + [
    dict(X=arr(6, 0)), dict(X=arr(-3, 4)), dict(X=arr(6, 4, ld=3)),
    dict(X=arr(6, 4, dtype=4)), dict(w=arr(1, 5, at=4 << 20)),
    dict(b=arr(2, 4, at=4 << 20)), dict(eps=-1.0), dict(eps=float("nan")),
    dict(act=6), dict(act=-1), dict(Y=arr(5, 4, at=2 << 20)),
    dict(Y=arr(6, 4, at=(1 << 20) + 4)), dict(Y=arr(6, 4, ld=5)),
    dict(w=arr(1, 4, at=2 << 20)), dict(b=arr(1, 4, at=2 << 20)),
    dict(mean=18), dict(rstd=17), dict(mean=32, rstd=32), dict(device=-1),
    # statistics (2 samples of 2 groups: 16 bytes each) in one another, in the
    # values before them and in the outputs
    dict(mean=32, rstd=44), dict(mean=44, rstd=32),
    dict(mean=(1 << 20) + 92), dict(rstd=(2 << 20) - 12),
    dict(rstd=4 << 20, w=arr(1, 4, at=4 << 20)),
    dict(work=24),
    # chunks of few large samples need a workspace
    dict(X=arr(1 << 20, 4, at=1 << 30), positions=1 << 20,
         Y=arr(1 << 20, 4, at=2 << 30), work=None)])
def test_group_norm_refusals(kw):
    assert group(**kw) == INV
    assert nv.svm_last_error()


_SAME = object()


def group_back(dY=None, X=_SAME, positions=3, groups=2, mean=16, rstd=16,
               w=None, b=None, act=0, res=None, dX=_SAME, dw=_SAME, db=_SAME,
               work=16, nbytes=1 << 40, device=0):
    d = lambda v, w: w if v is _SAME else v  # noqa: E731
    dY, X = dY or arr(6, 4), d(X, arr(6, 4, at=2 << 20))
    dX, dw, db = (d(dX, arr(6, 4, at=3 << 20)), d(dw, arr(1, 4, at=4 << 20)),
                  d(db, arr(1, 4, at=5 << 20)))
    return nv.load().svm_group_norm_backward(
        ref(dY), ref(X), positions, groups, mean, rstd, ref(w), ref(b), act,
        ref(res), ref(dX), ref(dw), ref(db), work, nbytes, device, None)


@pytest.mark.parametrize("kw", GROUPS + [
    dict(X=None), dict(X=arr(6, 5, at=2 << 20)), dict(mean=None),
    dict(rstd=None), dict(mean=18), dict(act=9), dict(dY=arr(6, 0)),
    dict(w=arr(2, 4, at=9 << 20)), dict(b=arr(1, 3, at=9 << 20)),
    dict(res=arr(6, 5, at=9 << 20)), dict(dX=arr(6, 4, at=2 << 20)),
    dict(dX=arr(6, 4, at=4 << 20)), dict(dX=arr(6, 4, ld=5)),
    dict(dX=arr(6, 4, at=3 << 20, dtype=1)), dict(dw=arr(1, 4)),
    dict(dw=arr(1, 3, at=4 << 20)), dict(dw=arr(1, 4, at=5 << 20)),
    dict(db=arr(1, 4, at=2 << 20)), dict(w=arr(1, 4, at=4 << 20)),
    dict(b=arr(1, 4, at=5 << 20)), dict(work=None), dict(nbytes=16),
    dict(device=-1)])
def test_group_norm_backward_refusals(kw):
    assert group_back(**kw) == INV
    assert nv.svm_last_error()


@needs_no_gpu
def test_group_norm_accepted():
    none = nv.SVM_E_DEVICE
    assert group() == none
    assert group(Y=arr(6, 4)) == none                        # in place
    assert group(positions=1, groups=4, work=None) == none
    assert group(X=arr(0, 4, at=None), Y=arr(0, 4, at=None)) == none
    assert group_back() == none
    assert group_back(dX=arr(6, 4)) == none                  # on dY
    assert group_back(res=arr(6, 4, at=3 << 20)) == none     # on dX
    assert group_back(dw=None, db=None, work=None) == none


def test_group_norm_workspace():
    lib, n = nv.load(), ct.c_int64(-1)
    for f in (lib.svm_group_norm_workspace,
              lib.svm_group_norm_backward_workspace):
        assert f(6, 3, 4, 2, 0, None) == INV
        for bad in ((6, 4, 4, 2, 0), (6, 0, 4, 2, 0), (-3, 3, 4, 2, 0),
                    (6, 3, 4, 3, 0), (6, 3, 0, 1, 0), (6, 3, 4, 2, 3)):
            assert f(*bad, ct.byref(n)) == INV and n.value == 0
        # every cut of the largest and the smallest
        for rows, per, cols, groups in (
                (0, 1, 1, 1), (1, 1, 1, 1), ((1 << 31) - 1, (1 << 31) - 1, 8,
                                             1), ((1 << 31) - 1, 1, 8, 8),
                (1, 1, 1 << 21, 1), (1, 1, 1 << 21, 1 << 21)):
            for t in range(3):
                assert f(rows, per, cols, groups, t, ct.byref(n)) == 0
                assert 0 <= n.value <= 1 << 36


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
    # what the binding packs: an address, a length and a type of 8 bytes
    assert got == [24, 8, 16]
