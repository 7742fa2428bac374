"""32-bit products whose sums are not finite: signs of infinities and places
of NaN as the formula gives them, at a bounded cost."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_layers import DEV, close, linear64

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def check(got, A, B):
    """got against A B^T: finite where that is, the same infinities, NaN
    where it is NaN."""
    want = A.double() @ B.double().t()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf)
    assert torch.equal(got.double()[inf], want[inf])
    fine = torch.isfinite(want)
    zero = lambda x: torch.nan_to_num(x, 0.0, 0.0, 0.0)  # noqa: E731
    A, B = zero(A), zero(B)
    y, _, _, tz = linear64(A, B, None, None, "none")
    # (values below 2^-109 are held to within 2^-134)
    tz = tz + 2.0 ** -134 * (A.double().abs().sum(1)[:, None]
                             + B.double().abs().sum(1))
    close(torch.where(fine, got, 0), torch.where(fine, y, 0), tz, "f32")


# few rows; tiles of every size; parts of a long summed index
SHAPES = [(3, 130, 70), (29, 2100, 40), (70, 64, 66), (130, 333, 257),
          (300, 45, 520), (5000, 72, 90), (40000, 40, 24)]


def planted(m, k, n, strided):
    g = torch.Generator(device=DEV).manual_seed(m)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    if strided:
        X, W, G = r(m, k + 3)[:, 1:k + 1], r(n, k + 1)[:, :k], r(m, n + 5)[:, :n]
    else:
        X, W, G = r(m, k), r(n, k), r(m, n)
    W[5] = 1.0              # every part of these but the first is 0
    W[6, 3] = 0.0           # infinity times zero: NaN
    X[0, 3] = INF
    X[m // 2, k - 1] = -INF
    X[m - 1, k // 2] = NAN
    W[n - 1, 1] = INF
    X[:, 1] = 2.0 ** -140   # infinity, not NaN
    return X, W, G


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_infinities_and_nan(m, k, n, strided):
    X, W, G = planted(m, k, n, strided)
    check(nv.svm_linear(X, W), X, W)
    G[1, 2] = -INF
    dX, dW, _ = nv.svm_linear_backward(G, X, W)
    check(dX, G, W.t())
    check(dW, G.t(), X.t())


def test_sums_past_the_largest():
    # products and sums that overflow: infinities, and NaN where two meet
    X = torch.full((70, 64), 1e38, device=DEV)
    W = torch.ones(66, 64, device=DEV)
    W[3] = -1.0
    W[4, :] = 0.0
    W[4, 63] = 3.0
    X[7, :32] = 2e38
    X[7, 32:] = -2e38
    Y = nv.svm_linear(X, W)
    assert bool((Y[:7, :3] == INF).all()) and bool((Y[:7, 3] == -INF).all())
    assert torch.allclose(Y[:7, 4], 3 * X[:7, 63])
    assert not bool(torch.isfinite(Y[7, 0]))


def timed(f):
    for _ in range(3):
        f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(5):
        f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / 5


@pytest.mark.parametrize("m", [20, 8192])
def test_nan_costs_a_few_times_the_call(m):
    # (formed one by one, each over the whole summed index, such sums took a
    # thousand times the call)
    k = n = 256
    X, W = torch.randn(m, k, device=DEV), torch.randn(n, k, device=DEV)
    G = torch.randn(m, n, device=DEV)
    call = lambda: nv.svm_linear_backward(G, X, W) + (  # noqa: E731
        nv.svm_linear(X, W),)
    fine = timed(call)
    X[:, 3] = NAN
    W[:, 5] = INF
    G[2] = NAN
    bad = timed(call)
    assert bad < 20 * fine, (bad, fine)
