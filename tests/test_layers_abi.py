"""Argument checks of the feature-map calls: every refusal comes before any
device call, so these run without a GPU (the pointers are never followed)."""
import ctypes as ct
import os

import numpy as np
import pytest

from paper_1706_05544_amd import native as nv

INV, UNS = nv.SVM_E_INVALID, nv.SVM_E_UNSUPPORTED


def arr(rows, cols, at=1 << 20, ld=None, dtype=nv.SVM_F32, dev=1):
    return nv.svm_array(at, rows, cols, cols if ld is None else ld, dtype,
                        dev)


def ref(a):
    return None if a is None else ct.byref(a)


def linear(X=None, W=None, b=None, R=None, act=0, Y=None, Z=None, work=16,
           nbytes=1 << 40, device=0, **kw):
    a = dict(X=arr(6, 4), W=arr(5, 4, at=2 << 20), b=None, R=None,
             Y=arr(6, 5, at=3 << 20), Z=None)
    for k, v in dict(X=X, W=W, b=b, R=R, Y=Y, Z=Z).items():
        if v is not None:
            a[k] = v
    for k in kw:  # null_X=True and so on
        a[k[5:]] = None
    return nv.load().svm_linear(ref(a["X"]), ref(a["W"]), ref(a["b"]),
                                ref(a["R"]), act, ref(a["Y"]), ref(a["Z"]),
                                work, nbytes, device, None)


@pytest.mark.parametrize("kw,code", [
    (dict(null_X=True), INV),
    (dict(null_W=True), INV),
    (dict(null_Y=True), INV),
    (dict(act=6), INV),
    (dict(act=-1), INV),
    (dict(X=arr(-1, 4)), INV),
    (dict(X=arr(1 << 31, 4)), INV),
    (dict(X=arr(6, 0)), INV),
    (dict(X=arr(6, (1 << 22) + 1)), INV),
    (dict(X=arr(6, 4, ld=3)), INV),
    (dict(X=arr(6, 4, ld=1 << 41)), INV),
    (dict(X=arr(6, 4, at=None)), INV),
    (dict(X=arr(6, 4, at=(1 << 20) + 2)), INV),
    (dict(X=arr(6, 4, dtype=3)), INV),
    (dict(X=arr(6, 4, dtype=nv.SVM_F16)), INV),
    (dict(X=arr(6, 4, dev=0)), UNS),
    (dict(W=arr(5, 3)), INV),
    (dict(W=arr(0, 4)), INV),
    (dict(b=arr(1, 6, at=4 << 20)), INV),
    (dict(b=arr(5, 1, at=4 << 20)), INV),
    (dict(R=arr(6, 4, at=4 << 20)), INV),
    (dict(Y=arr(6, 6, at=3 << 20)), INV),
    (dict(Z=arr(5, 5, at=4 << 20)), INV),
    # outputs on inputs, or on each other
    (dict(Y=arr(6, 5)), INV),
    (dict(Y=arr(6, 5, at=(2 << 20) + 16)), INV),
    (dict(Z=arr(6, 5, at=3 << 20)), INV),
    (dict(R=arr(6, 5, at=(3 << 20) + 20)), INV),
    (dict(R=arr(6, 5, at=3 << 20, ld=7)), INV),
    (dict(device=-1), INV),
    (dict(work=17), INV),
])
def test_linear_refusals(kw, code):
    assert linear(**kw) == code
    assert nv.svm_last_error()


def no_gpu(rc):
    # accepted by every check: the device is what is missing here
    return rc == nv.SVM_E_DEVICE


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="a GPU is present")
def test_accepted_arguments_reach_the_device_check():
    assert no_gpu(linear())
    assert no_gpu(linear(R=arr(6, 5, at=3 << 20)))      # residual in place
    # columns side by side in the rows of one buffer do not overlap
    assert no_gpu(linear(X=arr(6, 4, ld=9), Y=arr(6, 5, at=(1 << 20) + 16,
                                                  ld=9)))
    assert linear(X=arr(6, 4, ld=9),
                  Y=arr(6, 5, at=(1 << 20) + 12, ld=9)) == INV
    assert no_gpu(backward())
    assert no_gpu(backward(dX=None, X=arr(6, 4), W=None))
    assert no_gpu(norm())
    assert no_gpu(norm(Y=arr(6, 4)))                    # in place
    assert no_gpu(norm_backward())
    assert no_gpu(hinge())
    assert no_gpu(adamw())


_SAME = object()


def backward(dY=_SAME, X=_SAME, W=_SAME, Z=None, act=0, dX=_SAME, dW=_SAME,
             db=_SAME, work=16, nbytes=1 << 40):
    d = lambda v, w: w if v is _SAME else v  # noqa: E731
    dY, X, W = (d(dY, arr(6, 5)), d(X, arr(6, 4, at=2 << 20)),
                d(W, arr(5, 4, at=3 << 20)))
    dX, dW, db = (d(dX, arr(6, 4, at=4 << 20)), d(dW, arr(5, 4, at=5 << 20)),
                  d(db, arr(1, 5, at=6 << 20)))
    return nv.load().svm_linear_backward(
        ref(dY), ref(X), ref(W), ref(Z), act, ref(dX), ref(dW), ref(db),
        work, nbytes, 0, None)


@pytest.mark.parametrize("kw", [
    dict(dY=None), dict(X=None), dict(W=None), dict(act=2), dict(act=9),
    dict(dY=arr(6, 4)), dict(X=arr(5, 4)), dict(W=arr(5, 3)),
    dict(dX=arr(6, 3, at=4 << 20)), dict(dW=arr(4, 5, at=4 << 20)),
    dict(db=arr(1, 4, at=4 << 20)), dict(Z=arr(6, 4), act=1),
    dict(dX=arr(6, 4, at=2 << 20)), dict(dW=arr(5, 4, at=3 << 20)),
    dict(db=arr(1, 5)), dict(dX=arr(6, 4, at=5 << 20)),
    dict(dW=arr(5, 4, at=5 << 20, dtype=1)),
    # (with an activation dZ needs a workspace)
    dict(act=1, Z=arr(6, 5, at=7 << 20), work=None, nbytes=0),
    dict(act=1, Z=arr(6, 5, at=7 << 20), nbytes=8)])
def test_linear_backward_refusals(kw):
    assert backward(**kw) == INV
    assert nv.svm_last_error()


def norm(X=None, w=None, eps=1e-5, Y=None):
    X, Y = X or arr(6, 4), Y or arr(6, 4, at=2 << 20)
    return nv.load().svm_layer_norm(ref(X), ref(w), None, eps, ref(Y), None,
                                    None, 0, None)


@pytest.mark.parametrize("kw", [
    dict(X=arr(6, 0)), dict(w=arr(1, 5, at=4 << 20)), dict(eps=-1.0),
    dict(eps=float("nan")), dict(Y=arr(5, 4, at=2 << 20)),
    dict(Y=arr(6, 4, at=(1 << 20) + 4)), dict(Y=arr(6, 4, ld=5)),
    dict(w=arr(1, 4, at=2 << 20))])
def test_layer_norm_refusals(kw):
    assert norm(**kw) == INV


def norm_backward(mean=16, w=None, res=None, dX=_SAME, dw=_SAME, work=16,
                  nbytes=1 << 40):
    dX = arr(6, 4, at=3 << 20) if dX is _SAME else dX
    dw = arr(1, 4, at=4 << 20) if dw is _SAME else dw
    dY, X = arr(6, 4), arr(6, 4, at=2 << 20)
    return nv.load().svm_layer_norm_backward(
        ref(dY), ref(X), mean, 16, ref(w), ref(res), ref(dX), ref(dw), None,
        work, nbytes, 0, None)


@pytest.mark.parametrize("kw", [
    dict(mean=None), dict(w=arr(2, 4, at=9 << 20)),
    dict(res=arr(6, 5, at=9 << 20)), dict(dX=arr(6, 4, at=2 << 20)),
    dict(dX=arr(6, 4, at=4 << 20)), dict(dw=arr(1, 4)),
    dict(dw=arr(1, 3, at=4 << 20)), dict(work=None), dict(nbytes=16)])
def test_layer_norm_backward_refusals(kw):
    assert norm_backward(**kw) == INV


def hinge(S=None, labels=16, scale=1.0, dS=None, loss=16, work=16,
          nbytes=1 << 40):
    S = S or arr(6, 4)
    return nv.load().svm_hinge_loss(ref(S), labels, scale, ref(dS), loss,
                                    work, nbytes, 0, None)


@pytest.mark.parametrize("kw", [
    dict(S=arr(6, 0)), dict(labels=None), dict(loss=None),
    dict(scale=float("inf")), dict(dS=arr(6, 3, at=2 << 20)),
    dict(dS=arr(6, 4, at=(1 << 20) + 4)),
    # (losses of few scores need no workspace)
    dict(S=arr(60000, 4), work=None), dict(S=arr(60000, 4), nbytes=4)])
def test_hinge_refusals(kw):
    assert hinge(**kw) == INV


def adamw(n=300, bits=8, step=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8,
          null_params=False, count=1, **fields):
    t = nv.svm_adamw_tensor(16, 32, None, 64, 80, 96, 112, n, 0, 0)
    if bits == 32:
        t.m_scale = t.v_scale = None
    for k, v in fields.items():
        setattr(t, k, v)
    p = nv.svm_adamw_params(lr, b1, b2, eps, 0.0, 1.0, step, bits)
    return nv.load().svm_adamw_step(
        ct.addressof(t) if count else None, abs(count) or 1,
        None if null_params else ct.byref(p), 0, None)


@pytest.mark.parametrize("kw", [
    dict(null_params=True), dict(count=0), dict(bits=16), dict(step=0),
    dict(lr=float("nan")), dict(b1=1.0), dict(b2=-0.1), dict(eps=-1.0),
    dict(n=-1), dict(n=1 << 41), dict(dtype=5), dict(grad_dtype=1),
    dict(dtype=1, grad_dtype=2), dict(master=16), dict(param=None),
    dict(grad=None), dict(m=None), dict(v=None), dict(m_scale=None),
    dict(v_scale=None), dict(bits=32, m_scale=96), dict(param=18),
    dict(bits=32, m=66), dict(m=72), dict(master=24, dtype=1, grad_dtype=1),
    dict(m_scale=98)])
def test_adamw_refusals(kw):
    assert adamw(**kw) == INV
    assert nv.svm_last_error()


def test_adamw_state_refusals():
    f = nv.load().svm_adamw_state
    assert f(16, 16, 16, 16, -1, 16, 16, 0, None) == INV
    assert f(None, 16, 16, 16, 5, 16, 16, 0, None) == INV
    assert f(16, 16, 16, None, 5, None, 16, 0, None) == INV


def test_workspace_sizes():
    lib, n = nv.load(), ct.c_int64(-1)
    X, W, dY = arr(6, 4), arr(5, 4, at=2 << 20), arr(6, 5, at=3 << 20)
    assert lib.svm_linear_workspace(ref(X), ref(W), None) == INV
    assert lib.svm_linear_workspace(ref(X), ref(arr(5, 3)), ct.byref(n)) == INV
    assert lib.svm_linear_workspace(ref(X), ref(W), ct.byref(n)) == 0
    assert n.value >= 0
    assert lib.svm_linear_backward_workspace(
        ref(dY), ref(X), ref(W), 2, ref(X), ref(W), None, ct.byref(n)) == 0
    assert n.value >= 6 * 5 * 4  # dZ at the least
    assert lib.svm_linear_backward_workspace(
        ref(dY), None, ref(W), 2, None, ref(W), None, ct.byref(n)) == INV
    assert lib.svm_layer_norm_backward_workspace(-1, 4, ct.byref(n)) == INV
    assert lib.svm_layer_norm_backward_workspace(9, 4, ct.byref(n)) == 0
    assert n.value >= 2 * 4 * 4
    assert lib.svm_hinge_loss_workspace(9, 0, ct.byref(n)) == INV
    assert lib.svm_hinge_loss_workspace(9, 3, ct.byref(n)) == 0


def test_struct_layouts_match_header(tmp_path):
    import subprocess
    prog = tmp_path / "layout.c"
    prog.write_text(r'''
#include <stdio.h>
#include <stddef.h>
#include "mi355svm.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu %zu\n", sizeof(svm_array),
         offsetof(svm_array, ld), offsetof(svm_array, on_device),
         sizeof(svm_adamw_tensor), offsetof(svm_adamw_tensor, n),
         offsetof(svm_adamw_tensor, grad_dtype), sizeof(svm_adamw_params),
         offsetof(svm_adamw_params, bits));
  return 0;
}
''')
    exe = tmp_path / "layout"
    inc = os.path.join(os.path.dirname(os.path.dirname(
        os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-std=c99", "-I", inc, str(prog), "-o", str(exe)],
                   check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True,
                         check=True).stdout
    A, T, P = nv.svm_array, nv.svm_adamw_tensor, nv.svm_adamw_params
    assert [int(x) for x in got.split()] == [
        ct.sizeof(A), A.ld.offset, A.on_device.offset, ct.sizeof(T),
        T.n.offset, T.grad_dtype.offset, ct.sizeof(P), P.bits.offset]
    # the table that the binding fills column by column is the same struct
    r = nv._ADAMW_ROW
    assert r.itemsize == ct.sizeof(T)
    for name, _ in T._fields_:
        assert r.fields[name][1] == getattr(T, name).offset


def test_host_tensors_are_refused_by_the_binding():
    import torch
    X = torch.zeros(4, 8)
    for call in (lambda: nv.svm_linear(X, X), lambda: nv.svm_layer_norm(X),
                 lambda: nv.svm_linear(np.zeros((4, 8)), X),
                 lambda: nv.svm_hinge_loss(X, X),
                 lambda: nv.svm_adamw_step([X], [X], X, X)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == UNS


def test_rows_of_strided_tensors():
    import torch
    t = torch.zeros(6, 10)
    assert nv._rows_of(t) == (6, 10, 10)
    assert nv._rows_of(t[:, 2:7]) == (6, 5, 10)
    assert nv._rows_of(t[::2, :4]) == (3, 4, 20)
    assert nv._rows_of(t.t()) is None
    assert nv._rows_of(t[0]) == (1, 10, 10)
    assert nv._rows_of(t[0, ::2]) is None
    assert nv._rows_of(torch.zeros(4)[None].expand(3, 4)) is None
    b = torch.zeros(3, 4, 8)
    assert nv._rows_of(b) == (12, 8, 8)
    assert nv._rows_of(b[:, :2]) is None
    assert nv._rows_of(b[..., :5]) == (12, 5, 8)
    assert nv._rows_of(b.transpose(0, 1)) is None
    assert nv._rows_of(b[:, 1]) == (3, 8, 32)
    assert nv._rows_of(b[1:2, :, :3]) == (4, 3, 8)
    assert nv._rows_of(torch.zeros(3, 0, 5)) == (0, 5, 5)
    assert nv._rows_of(torch.zeros(())) is None


@pytest.mark.parametrize("scale", [1e39, -1e39, 2e38, 1e300])
def test_hinge_scale_past_32_bits(scale):
    # (the slope 2 scale would be infinite, and NaN where the loss is 0)
    assert hinge(scale=scale) == INV
    assert nv.svm_last_error()
