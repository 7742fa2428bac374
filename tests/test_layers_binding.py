"""The Python binding of the feature-map calls, without a GPU: CPU tensors
and a library that only records its calls stand in for the real ones."""
import pytest
import torch

from paper_1706_05544_amd import native as nv


class Recorded(nv._Call):
    """A call whose arrays may lie in host memory, and which knows what was
    copied after its stream began to wait for torch's."""

    late: list = []

    def __init__(self, t, stream):
        nv._DTYPES.update({torch.float32: nv.SVM_F32,
                           torch.bfloat16: nv.SVM_BF16,
                           torch.float16: nv.SVM_F16})
        self.device, self.index = t.device, t.get_device()
        self.stream, self.handle, self.other = stream, 0, False
        self.keep, self.waited = [], False

    def arr(self, t, what, out=False):
        a = super().arr(t, what, out)
        if self.waited and a is not None and a.data != t.data_ptr():
            self.late.append(what)
        return a

    def floats(self, t, rows, what):
        c = t.contiguous()
        if self.waited and c is not t:
            self.late.append(what)
        self.keep.append(c)
        return c.data_ptr()

    def ready(self):
        self.waited = True


class Library:
    """Accepts every call."""

    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def late(monkeypatch):
    monkeypatch.setattr(nv, "_Call", Recorded)
    monkeypatch.setattr(nv, "load", Library)
    monkeypatch.setattr(Recorded, "late", [])
    return Recorded.late


def test_inputs_are_copied_before_the_stream_waits(late):
    # a copy of an input without a row layout is queued on torch's stream:
    # another stream waits for it only if it is queued before the wait
    m, k, n = 6, 8, 10
    x = lambda rows, cols: torch.randn(cols, rows).t()  # noqa: E731
    v = lambda cols: torch.randn(2 * cols)[::2]  # noqa: E731
    nv.svm_linear(x(m, k), x(n, k), v(n), x(m, n), act="gelu", save=True)
    nv.svm_linear_backward(x(m, n), x(m, k), x(n, k), x(m, n), act="gelu")
    nv.svm_layer_norm(x(m, n), v(n), v(n), save=True)
    nv.svm_layer_norm_backward(x(m, n), x(m, n), v(m), v(m), v(n),
                               residual=x(m, n))
    nv.svm_hinge_loss(x(m, n), torch.zeros(2 * m, dtype=torch.int32)[::2])
    p = [torch.randn(n, k), torch.randn(n)]
    nv.svm_adamw_step(p, [x(n, k), v(n)], *nv.svm_adamw_states(p, bits=8))
    assert late == []


def test_what_is_written_in_place_is_seen_as_changed(late):
    # a tensor that autograd saved and a call then wrote over: its gradient
    # would come from the new values without a word
    def stale(*written):
        a = torch.ones((), requires_grad=True)
        return [(a * x).sum() for x in written]

    X, W, out = torch.ones(4, 6), torch.ones(5, 6), torch.ones(4, 5)
    p = [torch.ones(5, 6), torch.ones(5)]
    st = nv.svm_adamw_states(p, bits=8)
    st32 = nv.svm_adamw_states(p, bits=32)
    for written, call in (
            ([out], lambda: nv.svm_linear(X, W, out=out)),
            ([X], lambda: nv.svm_layer_norm(X, out=X)),
            (p, lambda: nv.svm_adamw_step(p, [x.clone() for x in p], *st)),
            ([*p, st32[0], st32[1]], lambda: nv.svm_adamw_step(
                p, [x.clone() for x in p], *st32))):
        losses = stale(*written)
        call()
        for loss in losses:
            with pytest.raises(RuntimeError, match="modified by an inplace"):
                loss.backward()
    before = [x._version for x in st[:4]]
    nv.svm_adamw_step(p, [x.clone() for x in p], *st)
    assert [x._version > b for x, b in zip(st, before)] == [True] * 4
    # and what is only read is not
    a = torch.ones((), requires_grad=True)
    loss = (a * X).sum() + (a * W).sum()
    nv.svm_linear(X, W)
    nv.svm_layer_norm(X)
    loss.backward()


def test_parameters_that_require_gradients_are_updated(late):
    p = [torch.nn.Parameter(torch.ones(5, 6))]
    nv.svm_adamw_step(p, [torch.ones(5, 6)], *nv.svm_adamw_states(p))
    with torch.inference_mode():
        x = torch.ones(3, 6)
        nv.svm_layer_norm(x, out=x)
    nv.svm_layer_norm(x, out=x)


def test_gradients_without_the_factor_that_they_do_not_need(late):
    dY, X, W = torch.ones(3, 2, 5), torch.ones(3, 2, 7), torch.ones(5, 7)
    dX, dW, db = nv.svm_linear_backward(dY, None, W, need=(True, False, True))
    assert dX.shape == X.shape and dW is None and db.shape == (5,)
    dX, dW, db = nv.svm_linear_backward(dY, X, None, need=(False, True, True))
    assert dX is None and dW.shape == W.shape and db.shape == (5,)
    dX, dW, db = nv.svm_linear_backward(dY, None, None,
                                        need=(False, False, True))
    assert dX is None and dW is None and db.shape == (5,)
    for args in ((None, W), (X, None)):
        with pytest.raises(nv.SvmError) as e:
            nv.svm_linear_backward(dY, *args)
        assert e.value.status == nv.SVM_E_INVALID
