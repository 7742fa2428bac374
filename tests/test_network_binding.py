"""The Python binding of the calls around a feature network's step and its
serving, without a GPU: CPU tensors and a library that only records its calls
stand in for the real ones."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_layers_binding import late  # noqa: F401 (a fixture)


@pytest.fixture(autouse=True)
def sizes_forgotten():
    # (workspace sizes that the stand-in library gave are not to stay)
    yield
    nv._group_norm_bytes.cache_clear()


def rows(m, n):
    return torch.randn(n, m).t()


def vec(n):
    return torch.randn(2 * n)[::2]


def packed(n, k, group=32):
    return nv.PackedWeights(torch.zeros(1 << 12, dtype=torch.uint8), (n, k),
                            group, torch.float32)


def test_inputs_are_copied_before_the_stream_waits(late):  # noqa: F811
    # a copy of an input without a row layout is queued on torch's stream:
    # another stream waits for it only if it is queued before the wait
    m, k, n = 6, 8, 10
    nv.svm_group_norm(rows(m, n), 5, vec(n), vec(n), act="silu", save=True)
    nv.svm_group_norm_backward(rows(m, n), rows(m, n), 5, rows(m, 5),
                               rows(m, 5), vec(n), vec(n),
                               residual=rows(m, n))
    nv.svm_pack_weights(rows(n, k), 32)
    nv.svm_linear_packed(rows(m, k), packed(n, k), vec(n), rows(m, n))
    p = [torch.randn(n, k), torch.randn(n)]
    nv.svm_grad_norm([rows(n, k), vec(n)], 1.0)
    nv.svm_adamw_step(p, [rows(n, k), vec(n)], *nv.svm_adamw_states(p),
                      factor=torch.ones(2)[::2])
    assert late == []


def test_what_is_written_in_place_is_seen_as_changed(late):  # noqa: F811
    def stale(x):
        return (torch.ones((), requires_grad=True) * x).sum()

    X, out, y = torch.ones(4, 6), torch.ones(4, 6), torch.ones(4, 5)
    p = [torch.ones(5, 6)]
    st = nv.svm_adamw_states(p)
    for x, call in (
            (out, lambda: nv.svm_group_norm(X, 2, out=out)),
            (X, lambda: nv.svm_group_norm(X, 2, out=X)),
            (y, lambda: nv.svm_linear_packed(X, packed(5, 6), out=y)),
            (p[0], lambda: nv.svm_adamw_step(p, [p[0].clone()], *st,
                                             factor=torch.ones(())))):
        loss = stale(x)
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace"):
            loss.backward()
    # and what is only read is not
    a = torch.ones((), requires_grad=True)
    loss = (a * X).sum()
    nv.svm_group_norm(X, 2)
    nv.svm_linear_packed(X, packed(5, 6))
    nv.svm_pack_weights(X, 32)
    nv.svm_grad_norm([X])
    loss.backward()


def test_shapes_and_what_is_asked_for(late):  # noqa: F811
    X = torch.ones(3, 4, 2, 6)
    Y, mean, rstd = nv.svm_group_norm(X, 3, save=True)
    assert Y.shape == X.shape and mean.shape == rstd.shape == (3, 3)
    dX, dw, db = nv.svm_group_norm_backward(X, X, 3, mean, rstd,
                                            need=(False, True, False))
    assert dX is None and dw.shape == (6,) and db is None
    assert nv.svm_linear_packed(X, packed(5, 6)).shape == (3, 4, 2, 5)
    assert nv._positions(X) == 8 and nv._positions(torch.ones(3, 6)) == 1
    norm, factor = nv.svm_grad_norm([X])
    assert norm.shape == factor.shape == ()
    assert norm.dtype == factor.dtype == torch.float32
    W = nv.svm_unpack_weights(packed(5, 6))
    assert W.shape == (5, 6) and W.dtype == torch.float32


def test_refusals_of_the_binding(late):  # noqa: F811
    X, st = torch.ones(4, 6), torch.ones(4, 2)
    for call in (lambda: nv.svm_group_norm(X[0], 2),
                 lambda: nv.svm_group_norm_backward(X, X[:3], 2, st, st),
                 lambda: nv.svm_group_norm_backward(X, X, 2, st, st[:3]),
                 lambda: nv.svm_linear_packed(X, X),
                 lambda: nv.svm_unpack_weights(X),
                 lambda: nv.svm_grad_norm([]),
                 lambda: nv.svm_grad_norm([X, 3.0]),
                 lambda: nv.PackedWeights(X, (5, 6), 32, torch.float32),
                 lambda: nv.PackedWeights(torch.zeros(9, dtype=torch.uint8),
                                          (5,), 32, torch.float32)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == nv.SVM_E_INVALID
    with pytest.raises(nv.SvmError) as e:
        nv.svm_grad_norm([X.double()])
    assert e.value.status == nv.SVM_E_UNSUPPORTED


def test_host_tensors_are_refused():
    X = torch.zeros(4, 8)
    for call in (lambda: nv.svm_group_norm(X, 2),
                 lambda: nv.svm_group_norm_backward(X, X, 2, X, X),
                 lambda: nv.svm_pack_weights(X),
                 lambda: nv.svm_linear_packed(X, packed(4, 8)),
                 lambda: nv.svm_unpack_weights(packed(4, 8)),
                 lambda: nv.svm_grad_norm([X])):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == nv.SVM_E_UNSUPPORTED
