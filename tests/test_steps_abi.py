"""The AdamW step that counts the steps left out: argument checks, binding and
host side, without a GPU (no pointer is followed)."""
import ctypes as ct
import inspect
import os

import pytest
import torch

from paper_1706_05544_amd import build as b
from paper_1706_05544_amd import native as nv
from test_layers_binding import late  # noqa: F401 (a fixture)
from test_layers_host import run_driver
from test_network_abi import INV, needs_no_gpu

MB = 1 << 20


def counted(factor=30 * MB, left_out=31 * MB, null=False, bits=32, device=0,
            count=1, **fields):
    # 300 values: two blocks of states
    t = nv.svm_adamw_tensor(MB, 2 * MB, None, 3 * MB, 4 * MB, None, None, 300,
                            nv.SVM_BF16, nv.SVM_BF16)
    if bits == 8:
        t.m_scale, t.v_scale = 5 * MB, 6 * MB
    for k, v in fields.items():
        setattr(t, k, v)
    p = nv.svm_adamw_params(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 1, bits)
    return nv.load().svm_adamw_step_counted(
        ct.addressof(t), count, None if null else ct.byref(p), factor,
        left_out, device, None)


@pytest.mark.parametrize("kw", [
    dict(null=True), dict(n=-1), dict(param=None), dict(m=72), dict(dtype=5),
    dict(count=-1), dict(device=-1), dict(factor=30 * MB + 2),
    dict(left_out=31 * MB + 4), dict(factor=31 * MB),
    dict(factor=31 * MB + 4),
    # in the parameter, the states, their scales, the master copy
    dict(factor=MB), dict(factor=MB + 596), dict(left_out=MB + 592),
    dict(left_out=3 * MB + 2040), dict(factor=4 * MB + 2044),
    dict(left_out=3 * MB + 504, bits=8), dict(left_out=4 * MB, bits=8),
    dict(factor=5 * MB + 4, bits=8), dict(left_out=6 * MB, bits=8),
    dict(factor=7 * MB + 2044, master=7 * MB)])
def test_refusals(kw):
    assert counted(**kw) == INV
    assert nv.svm_last_error()


@needs_no_gpu
def test_accepted():
    for kw in (dict(), dict(factor=None), dict(left_out=None),
               dict(factor=None, left_out=None), dict(factor=2 * MB),
               dict(factor=MB + 600), dict(left_out=3 * MB + 2048),
               dict(left_out=3 * MB + 512, bits=8), dict(factor=MB, n=0),
               dict(factor=5 * MB + 8, bits=8), dict(count=0)):
        assert counted(**kw) == nv.SVM_E_DEVICE


def test_the_thread_keeps_its_device(tmp_path):
    run_driver(tmp_path, "steps_device_driver",
               [os.path.join(b.CSRC, "steps.cpp")])


def test_binding(late):  # noqa: F811
    p = [torch.randn(6, 8).t().contiguous(), torch.randn(5)]
    g = [torch.randn(6, 8).t(), torch.randn(10)[::2]]
    st = nv.svm_adamw_states(p)
    c = torch.zeros((), dtype=torch.int64)
    # inputs are copied before the stream waits, and the count is written
    version = c._version
    nv.svm_adamw_step(p, g, *st, factor=torch.ones(2)[::2], left_out=c)
    assert late == [] and c._version > version
    for bad in (0, torch.zeros(()), torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(nv.SvmError) as e:
            nv.svm_adamw_step(p, g, *st, left_out=bad)
        assert e.value.status == INV


def test_arguments_by_place(late):  # noqa: F811
    # the stream is the fifteenth, as before there was a factor
    p = [torch.ones(3)]
    st = nv.svm_adamw_states(p)
    nv.svm_adamw_step(p, [torch.ones(3)], *st, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1,
                      1.0, None, torch.ones(()))
    assert list(inspect.signature(nv.svm_adamw_step).parameters)[12:] == [
        "step", "grad_scale", "stream", "factor", "left_out"]
