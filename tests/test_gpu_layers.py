"""The feature-map operators against their definitions in 64 bits.

Tolerances come from the formats and the sums, not from results.  u is half
a unit in the last place of the type (2^-24, 2^-8, 2^-11: 24, 8 and 11 bits).  A sum of K terms
that is held in 32 bits is off by at most about K 2^-23 of the sum of the
terms' magnitudes (2^-23 and not 2^-24: the matrix instructions need not
round each addition to nearest), and so are the products of 32-bit factors
in three parts, whose dropped terms are below 3 2^-24 of each product.  The
activations are Lipschitz with at most 1.13, and their own evaluation is good
to a few units of 2^-24 (1 + z^2) (the argument of exp is rounded).  A
gradient that passes through dZ in a 16-bit type is off by u of each term.
"""
import math

import numpy as np
import pytest
import torch

from paper_1706_05544_amd import native as nv

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# below the normal range a type is off by half its smallest step
FLOOR = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
ACTS = ("none", "relu", "gelu", "silu", "tanh", "cos")
E = 2.0 ** -23


def act64(name, z):
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(
            2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "tanh":
        y = torch.tanh(z)
        return y, 1 - y * y
    if name == "cos":
        return torch.cos(z), -torch.sin(z)
    return z, torch.ones_like(z)


def rnd(g, *shape, by=1.0, t="f32"):
    return (torch.randn(*shape, generator=g) * by).to(DEV).to(TYPES[t])


def gen(*key):
    return torch.Generator().manual_seed(hash(tuple(key)) % (1 << 31)
                                         if all(isinstance(x, int)
                                                for x in key) else 7)


def close(got, want, tol, t):
    """Within tol (before the last rounding) and the rounding to the type."""
    want = want.double()
    lim = tol + U[t] * want.abs() * (1 + 1e-6) + U[t] * tol + FLOOR[t]
    bad = (got.double() - want).abs() > lim
    # a value within tol of the type's largest may round to infinity
    assert got.shape == want.shape
    assert not bool(bad.any()), (
        float(((got.double() - want).abs() / lim).max()), int(bad.sum()))


def linear64(X, W, b, R, act):
    X, W = X.double(), W.double()
    z = X @ W.t()
    mag = X.abs() @ W.abs().t()
    if b is not None:
        z = z + b.double()
        mag = mag + b.double().abs()
    y, _ = act64(act, z)
    tz = (X.shape[1] + 8) * E * mag
    ty = 1.13 * tz + 4 * E * (1 + z * z)
    if R is not None:
        y = y + R.double()
        ty = ty + E * (y.abs() + R.double().abs())
    return y, z, ty, tz


def check_linear(X, W, b, R, act, t, save=True, **kw):
    got = nv.svm_linear(X, W, b, R, act=act, save=save, **kw)
    Y, Z = got if save else (got, None)
    y, z, ty, tz = linear64(X, W, b, R, act)
    close(Y, y, ty, t)
    if save:
        close(Z, z, tz, t)
    return Y, Z


# sizes on both sides of every tile edge, and of the choice between kernels
SIZES = [(1, 1, 1), (1, 784, 1024), (3, 5, 7), (2, 2049, 40), (16, 64, 64),
         (17, 130, 65), (33, 8, 129), (64, 64, 64), (65, 63, 257),
         (128, 256, 128), (129, 257, 127), (255, 72, 256), (257, 1001, 513),
         (300, 501, 333), (1000, 128, 10), (513, 520, 1)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear(m, k, n, t):
    g = gen(m, k, n)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
    b, R = rnd(g, n, t=t), rnd(g, m, n, t=t)
    check_linear(X, W, b, R, "gelu", t)
    check_linear(X, W, None, None, "none", t, save=False)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,k,n", [(5, 40, 24), (130, 72, 200)])
def test_linear_acts(m, k, n, act, t):
    g = gen(m, k, n)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=2 * k ** -0.5, t=t)
    b, R = rnd(g, n, t=t), rnd(g, m, n, t=t)
    check_linear(X, W, b, R, act, t)
    check_linear(X, W, b, None, act, t, save=False)
    check_linear(X, W, None, R, act, t)


# large enough for the largest tiles, with edges in every direction
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", [(4096, 512, 4096), (4161, 200, 4090),
                                   (20000, 96, 1030)])
def test_linear_large(m, k, n, t):
    g = torch.Generator(device=DEV).manual_seed(m + k + n)
    X = torch.randn(m, k, generator=g, device=DEV).to(TYPES[t])
    W = (torch.randn(n, k, generator=g, device=DEV) * k ** -0.5).to(TYPES[t])
    b = torch.randn(n, generator=g, device=DEV).to(TYPES[t])
    R = torch.randn(m, n, generator=g, device=DEV).to(TYPES[t])
    check_linear(X, W, b, R, "gelu", t)


def grads64(dY, X, W, Z, act, t):
    dY, X, W = dY.double(), X.double(), W.double()
    dz = dY
    tz = torch.zeros_like(dY)
    if act != "none":
        z = Z.double()
        dz = dY * act64(act, z)[1]
        tz = dY.abs() * 4 * E * (1 + z * z)
    m, n = dY.shape
    part = tz + (0 if t == "f32" else U[t] + E) * dz.abs()
    if t != "f32":
        part = part + FLOOR[t]
    return ((dz @ W, (n + 8) * E * (dz.abs() @ W.abs())
             + part @ W.abs()),
            (dz.t() @ X, (m + 8) * E * (dz.abs().t() @ X.abs())
             + part.t() @ X.abs()),
            (dz.sum(0), (m + 8) * E * dz.abs().sum(0) + tz.sum(0)))


def check_linear_backward(dY, X, W, Z, act, t, need=(True, True, True)):
    got = nv.svm_linear_backward(dY, X, W, Z, act=act, need=need)
    for x, (want, tol), asked in zip(got, grads64(dY, X, W, Z, act, t), need):
        assert (x is not None) == asked
        if asked:
            close(x, want, tol, t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear_backward(m, k, n, t):
    g = gen(m, k, n, 1)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
    dY, Z = rnd(g, m, n, t=t), rnd(g, m, n, t=t)
    check_linear_backward(dY, X, W, Z, "gelu", t)
    check_linear_backward(dY, X, W, None, "none", t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
def test_linear_backward_acts(act, t):
    m, k, n = 70, 40, 96
    g = gen(m, k, n, 2)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
    dY, Z = rnd(g, m, n, t=t), rnd(g, m, n, by=2.0, t=t)
    Z[0, :3] = 0.0  # relu's slope at 0 is 0
    check_linear_backward(dY, X, W, Z, act, t)
    for need in ((True, False, False), (False, True, False),
                 (False, False, True), (False, True, True)):
        check_linear_backward(dY, X, W, Z, act, t, need)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", [(4096, 1024, 1536), (20000, 128, 200),
                                   (6897, 501, 333), (100003, 30, 40)])
def test_linear_backward_large(m, k, n, t):
    g = torch.Generator(device=DEV).manual_seed(m + k + n)
    X = torch.randn(m, k, generator=g, device=DEV).to(TYPES[t])
    W = (torch.randn(n, k, generator=g, device=DEV) * k ** -0.5).to(TYPES[t])
    dY = torch.randn(m, n, generator=g, device=DEV).to(TYPES[t])
    Z = torch.randn(m, n, generator=g, device=DEV).to(TYPES[t])
    check_linear_backward(dY, X, W, Z, "silu", t)


def directional(f, x, d, h=1e-5):
    """Central difference of the scalar f along d, in 64 bits."""
    return float((f(x + h * d) - f(x - h * d)) / (2 * h))


@pytest.mark.parametrize("act", ACTS)
def test_linear_gradient_against_differences(act):
    m, k, n = 9, 11, 6
    g = gen(m, k, n, 3)
    X, W, b, dY = (rnd(g, m, k), rnd(g, n, k, by=0.3), rnd(g, n),
                   rnd(g, m, n))
    _, Z = nv.svm_linear(X, W, b, act=act, save=True)
    dX, dW, db = nv.svm_linear_backward(dY, X, W, Z, act=act)
    x, w, c, gy = X.double(), W.double(), b.double(), dY.double()

    def loss(x=x, w=w, c=c):
        return (gy * act64(act, x @ w.t() + c)[0]).sum()

    for name, v, got in (("x", x, dX), ("w", w, dW), ("c", c, db)):
        d = torch.randn(v.shape, generator=g).to(DEV).double()
        want = directional(lambda u: loss(**{name: u}), v, d)
        have = float((got.double() * d).sum())
        # 32-bit gradients of some 60 terms of order 1 each, against a
        # difference whose own error is of order h^2 + 2^-52 / h
        lim = float((got.double().abs() * d.abs()).sum()) * 100 * E + 1e-6
        assert abs(have - want) <= lim, (name, have, want)


@pytest.mark.parametrize("t", list(TYPES))
def test_linear_strides(t):
    # columns of wider buffers, rows at odd addresses, a transposed weight
    g = gen(4, 5)
    m, k, n = 77, 100, 90
    for shift in (0, 1, 3, 8):
        XB, RB = rnd(g, m, k + 29, t=t), rnd(g, m, n + 13, t=t)
        X, R = XB[:, shift:shift + k], RB[:, shift:shift + n]
        W = rnd(g, k, n, by=0.1, t=t).t()
        b = rnd(g, 2 * n, t=t)[::2]
        out = torch.full((m, n + 11), 7.0, dtype=TYPES[t], device=DEV)
        y, _, ty, _ = linear64(X, W, b, R, "tanh")
        got = nv.svm_linear(X, W, b, R, act="tanh",
                            out=out[:, shift:shift + n])
        close(got, y, ty, t)
        # nothing beside the output is written
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[:, shift:shift + n] = False
        assert bool((out[rest] == 7.0).all())
        dYB, ZB = rnd(g, m, n + 9, t=t), rnd(g, m, n + 5, t=t)
        check_linear_backward(dYB[:, shift:shift + n], X, W,
                              ZB[:, 3:3 + n], "silu", t)


@pytest.mark.parametrize("t", list(TYPES))
def test_linear_in_place_residual_and_leading_dims(t):
    g = gen(8, 8)
    X, W = rnd(g, 4, 33, 64, t=t), rnd(g, 128, 64, by=0.1, t=t)
    R = rnd(g, 4, 33, 128, t=t)
    want, _, tol, _ = linear64(X.reshape(-1, 64), W, None,
                               R.reshape(-1, 128), "relu")
    got = nv.svm_linear(X, W, None, R, act="relu", out=R)
    assert got is R and got.shape == (4, 33, 128)
    close(got.view(-1, 128), want, tol, t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m", [1, 40, 300])
def test_linear_not_finite_stays_in_its_row(m, t):
    # an infinity or a NaN in a row of X reaches that row of Y alone, with
    # the signs that the formula gives
    g = gen(m, 99)
    X, W = rnd(g, m, 96, t=t), rnd(g, 70, 96, t=t)
    W[5] = 1.0          # every part of these weights but the first is 0
    W[6, 3] = 0.0       # infinity times zero: NaN
    X[0, 3] = float("inf")
    if m > 1:
        X[m // 2, 10] = float("-inf")
        X[m - 1, 95] = float("nan")
    Y = nv.svm_linear(X, W)
    want = X.double() @ W.double().t()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(Y), torch.isnan(want))
    assert torch.equal(torch.isfinite(Y), fine)
    inf = torch.isinf(want)
    assert torch.equal(Y.double()[inf], want[inf])
    y, _, ty, _ = linear64(torch.nan_to_num(X, 0.0, 0.0, 0.0), W, None, None,
                           "none")
    close(torch.where(fine, Y, 0), torch.where(fine, y, 0), ty, t)


@pytest.mark.parametrize("m", [11, 66])  # few rows, and tiles
@pytest.mark.parametrize("act", ACTS)
def test_activations_at_the_ends_of_the_range(act, m):
    inf = float("inf")
    vals = [0.0, -0.0, 1e-30, -1e-30, 0.2, 30.0, -30.0, 88.0, -88.0, 1e4,
            -1e4] + [inf, -inf, float("nan"), 1e30, -1e30] * (m > 16)
    z = torch.tensor(vals, device=DEV)[:, None]
    X = torch.cat([z, torch.zeros(m - len(vals), 1, device=DEV)])
    W = torch.ones(3, 1, device=DEV)
    Y, Z = nv.svm_linear(X, W, act=act, save=True)
    assert torch.equal(torch.nan_to_num(Z, 7.0),
                       torch.nan_to_num(X.expand(m, 3), 7.0))
    G = torch.ones(m, 3, device=DEV)
    dX = nv.svm_linear_backward(G, X, W, Z, act=act,
                                need=(True, False, False))[0]
    x = X.double()
    y, d = act64(act, x)
    if act == "cos":  # angles past 1e8 are left open
        y, d = (torch.where(x.abs() > 1e8, 0, v) for v in (y, d))
        Y, dX = (torch.where(X.abs() > 1e8, 0, v) for v in (Y, dX))
    # (gelu and silu at -inf, and their slopes at both ends, are products of
    # an infinity with 0: NaN, as the formulas in 32 bits are)
    near = 4 * E * (1 + torch.nan_to_num(x, 0, 0, 0).clamp(-40, 40) ** 2
                    + torch.nan_to_num(y.abs(), 0, 0, 0))
    for got, want, tol in ((Y[:, :1], y, near), (dX, 3 * d, 8 * near)):
        fine = torch.isfinite(want)
        assert torch.equal(torch.isfinite(got), fine), (got, want)
        close(torch.where(fine, got, 0), torch.where(fine, want, 0),
              torch.where(fine, tol, 1), "f32")


def test_linear_32_bit_range():
    # factors near the ends of the 32-bit range: products that are fine stay
    # exact to 32 bits
    g = gen(12, 12)
    X, W = rnd(g, 70, 64), rnd(g, 66, 64)
    for a, b in ((2.0 ** 100, 2.0 ** -100), (2.0 ** 120, 2.0 ** -60),
                 (2.0 ** -60, 2.0 ** 40), (3.0e38 / 6, 2.0 ** -90)):
        check_linear(X * a, W * b, None, None, "none", "f32", save=False)


def test_linear_empty_rows():
    for t in TYPES.values():
        X = torch.empty(0, 20, dtype=t, device=DEV)
        W = torch.randn(30, 20, device=DEV).to(t)
        Y, Z = nv.svm_linear(X, W, save=True)
        assert Y.shape == Z.shape == (0, 30)
        dX, dW, db = nv.svm_linear_backward(Y, X, W, Z, act="gelu")
        assert dX.shape == (0, 20)
        assert not bool(dW.any()) and not bool(db.any())


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_linear_offsets_past_32_bits(t):
    # 1.2M x 2048 values: the last rows lie past 2^31 values and 2^32 bytes
    m, k, n = 1200007, 2048, 16
    X = torch.empty(m, k, dtype=TYPES[t], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    rows = torch.randn(4096, k, generator=g, device=DEV).to(TYPES[t])
    for i in range(0, m, 4096):
        X[i:i + 4096] = rows[:min(4096, m - i)]
    W = (torch.randn(n, k, generator=g, device=DEV) * k ** -0.5).to(TYPES[t])
    Y = nv.svm_linear(X, W)
    y, _, ty, _ = linear64(rows, W, None, None, "none")
    for i in (0, 1048576, m - 1 - (m - 1) % 4096):
        r = min(4096, m - i)
        close(Y[i:i + r], y[:r], ty[:r], t)
    # and its gradients: every row of dY is the same, dW the sum of X's rows
    dY = torch.zeros(m, n, dtype=TYPES[t], device=DEV)
    dY[-3:] = 1.0
    dX, dW, db = nv.svm_linear_backward(dY, X, W)
    xs = X[-3:].double()
    close(dW, xs.sum(0).expand(n, k), 16 * E * xs.abs().sum(0).expand(n, k), t)
    w = W.double()
    close(dX[-3:], w.sum(0).expand(3, k),
          (n + 8) * E * w.abs().sum(0).expand(3, k), t)
    assert not bool(dX[:-3].any())
    assert bool((db == 3.0).all())


def test_linear_more_rows_than_a_launch_has_threads_for():
    # 1.1e9 rows: 2^32 threads would not cover them in tiles of any size
    m = 1100000001
    X = torch.ones(m, 1, dtype=torch.bfloat16, device=DEV)
    X[-1] = 3.0
    X[1 << 30] = 5.0
    W = torch.tensor([[2.0]], dtype=torch.bfloat16, device=DEV)
    Y = nv.svm_linear(X, W)
    at = torch.tensor([0, 268435455, 268435456, 1 << 30, m - 2, m - 1],
                      device=DEV)
    assert Y[at, 0].tolist() == [2.0, 2.0, 2.0, 10.0, 2.0, 6.0]
    assert int((Y != 2.0).sum()) == 2


# ------------------------------------------------------------- layer norm


def norm64(X, w, b, eps):
    x = X.double()
    mu = x.mean(1, keepdim=True)
    d = x - mu
    rs = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    xh = d * rs
    y = xh * (1 if w is None else w.double()) + (0 if b is None
                                                 else b.double())
    return y, mu, rs, xh


NORM_SIZES = [(1, 1), (1, 784), (3, 2), (7, 64), (5, 127), (33, 128),
              (130, 501), (64, 1000), (9, 2048), (17, 4096), (5, 8191),
              (3, 12288), (2, 70001), (4000, 16), (70000, 24)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n", NORM_SIZES)
def test_layer_norm(m, n, t):
    g = torch.Generator(device=DEV).manual_seed(m * 31 + n)
    X = (3 * torch.randn(m, n, generator=g, device=DEV) + 5).to(TYPES[t])
    w = torch.randn(n, generator=g, device=DEV).to(TYPES[t])
    b = torch.randn(n, generator=g, device=DEV).to(TYPES[t])
    eps = 1e-3
    for ww, bb in ((w, b), (None, None), (w, None)):
        Y, mean, rstd = nv.svm_layer_norm(X, ww, bb, eps=eps, save=True)
        y, mu, rs, xh = norm64(X, ww, bb, eps)
        # the mean: a sum of n terms (held by many partial sums, at most 2 +
        # n / 64 long ones); the deviations inherit its error
        s = (n / 64 + 16) * E
        tm = s * X.double().abs().mean(1, keepdim=True)
        tr = 2 * s * rs + tm * rs * rs * 2
        tx = tm * rs + xh.abs() * tr / rs + 4 * E * xh.abs()
        close(mean[:, None], mu, tm, "f32")
        close(rstd[:, None], rs, tr, "f32")
        wa = 1 if ww is None else ww.double().abs()
        close(Y, y, tx * wa + 2 * E * y.abs() + 2 * E * (xh * wa).abs(), t)


def test_layer_norm_large_offset_and_constant_rows():
    # the second pass over the deviations: no cancellation for rows far from
    # 0, and a constant row gives the bias
    g = gen(5)
    X = rnd(g, 40, 300) + 3000.0
    X[7] = 2.5
    b = rnd(g, 300)
    Y, mean, rstd = nv.svm_layer_norm(X, None, b, eps=1e-5, save=True)
    y, mu, rs, xh = norm64(X, None, b, 1e-5)
    # the mean is good to E of 3000, which is the deviations' error
    tol = 3100 * 8 * E * rs * (1 + xh.abs())
    close(Y[:7], y[:7], tol[:7], "f32")
    close(Y[8:], y[8:], tol[8:], "f32")
    assert torch.equal(Y[7], b)
    assert float(mean[7]) == 2.5


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n", NORM_SIZES)
def test_layer_norm_backward(m, n, t):
    g = torch.Generator(device=DEV).manual_seed(m * 37 + n)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    X = (2 * r(m, n) + 1).to(TYPES[t])
    dY, w, res = r(m, n).to(TYPES[t]), r(n).to(TYPES[t]), r(m, n).to(TYPES[t])
    _, mu, rs, xh = norm64(X, None, None, 1e-3)
    mean, rstd = mu.float().view(-1), rs.float().view(-1)
    mu, rs = mean.double()[:, None], rstd.double()[:, None]
    x, dy = X.double(), dY.double()
    xh = (x - mu) * rs
    ex = 2 * E * (x.abs() + mu.abs()) * rs + 2 * E * xh.abs()  # of xh
    for ww, rr in ((w, res), (None, None)):
        a = dy * (1 if ww is None else ww.double())
        dx = rs * (a - a.mean(1, keepdim=True)
                   - xh * (a * xh).mean(1, keepdim=True))
        s = (n / 64 + 16) * E
        aa = a.abs()
        e1 = s * aa.mean(1, keepdim=True)
        e2 = (s * (aa * xh.abs()).mean(1, keepdim=True)
              + (aa * ex).mean(1, keepdim=True))
        tol = rs * (4 * E * aa + e1 + xh.abs() * e2
                    + ex * (aa * xh.abs()).mean(1, keepdim=True)
                    + 4 * E * (aa.mean(1, keepdim=True) + xh.abs()
                               * (aa * xh.abs()).mean(1, keepdim=True)))
        if rr is not None:
            dx = dx + rr.double()
            tol = tol + 2 * E * (dx.abs() + rr.double().abs())
        got = nv.svm_layer_norm_backward(dY, X, mean, rstd, ww, residual=rr)
        close(got[0], dx, tol, t)
        # sums over rows: partial sums of at most m terms each
        close(got[1], (dy * xh).sum(0),
              (m + 8) * E * (dy * xh).abs().sum(0) + (dy.abs() * ex).sum(0),
              t)
        close(got[2], dy.sum(0), (m + 8) * E * dy.abs().sum(0), t)
    only = nv.svm_layer_norm_backward(dY, X, mean, rstd, w,
                                      need=(False, True, False))
    assert only[0] is None and only[2] is None
    assert torch.equal(only[1], got[1])
    only = nv.svm_layer_norm_backward(dY, X, mean, rstd, None,
                                      need=(True, False, False))
    assert only[1] is None and torch.equal(only[0], got[0])


def test_layer_norm_gradient_against_differences():
    g = gen(21)
    m, n = 6, 13
    X, w, b, dY = rnd(g, m, n), rnd(g, n), rnd(g, n), rnd(g, m, n)
    _, mean, rstd = nv.svm_layer_norm(X, w, b, eps=0.01, save=True)
    dX, dw, db = nv.svm_layer_norm_backward(dY, X, mean, rstd, w)
    args = dict(x=X.double(), w=w.double(), b=b.double())

    def loss(**kw):
        v = {**args, **kw}
        return (dY.double() * norm64(v["x"], v["w"], v["b"], 0.01)[0]).sum()

    for name, got in (("x", dX), ("w", dw), ("b", db)):
        d = torch.randn(args[name].shape, generator=g).to(DEV).double()
        want = directional(lambda u: loss(**{name: u}), args[name], d)
        have = float((got.double() * d).sum())
        lim = float((got.double().abs() * d.abs()).sum()) * 200 * E + 1e-6
        assert abs(have - want) <= lim, (name, have, want)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n", [96, 501, 4096])
def test_layer_norm_strides_and_in_place(n, t):
    g = gen(n)
    m = 50
    for shift in (0, 1, 8):
        B = rnd(g, m, n + 24, t=t)
        X = B[:, shift:shift + n]
        y = nv.svm_layer_norm(X.contiguous())
        G = rnd(g, m, n + 3, t=t)[:, 1:1 + n]
        mean, rstd = nv.svm_layer_norm(X, save=True)[1:]
        want = nv.svm_layer_norm_backward(G.contiguous(), X.contiguous(),
                                          mean, rstd)
        got = nv.svm_layer_norm_backward(G, X, mean, rstd)
        for x, z in zip(got, want):
            # the same values in another order of addition
            lim = max(2.0 ** -7 if t == "bf16" else 2.0 ** -10 if t == "f16"
                      else 2.0 ** -18, 0) * z.double().abs().amax().item()
            assert float((x.double() - z.double()).abs().max()) <= lim
        beside = B.clone()
        nv.svm_layer_norm(X, out=X)
        lim = U[t] * 2 * y.double().abs() + 64 * E
        assert bool(((X.double() - y.double()).abs() <= lim).all())
        rest = torch.ones_like(B, dtype=torch.bool)
        rest[:, shift:shift + n] = False
        assert torch.equal(B[rest], beside[rest])


def test_layer_norm_not_finite_stays_in_its_row():
    g = gen(31)
    X = rnd(g, 20, 200)
    clean = nv.svm_layer_norm(X)
    X[3, 7], X[11, 199] = float("nan"), float("inf")
    Y = nv.svm_layer_norm(X)
    bad = torch.zeros(20, dtype=torch.bool, device=DEV)
    bad[3] = bad[11] = True
    assert torch.equal(Y[~bad], clean[~bad])
    assert bool(torch.isnan(Y[3]).all()) and bool(torch.isnan(Y[11]).all())


def test_layer_norm_no_rows():
    X = torch.empty(0, 40, device=DEV)
    Y, mean, rstd = nv.svm_layer_norm(X, save=True)
    assert Y.shape == (0, 40) and mean.numel() == 0
    dX, dw, db = nv.svm_layer_norm_backward(X, X, mean, rstd)
    assert dX.shape == (0, 40)
    assert not bool(dw.any()) and not bool(db.any()) and dw.shape == (40,)


def test_layer_norm_offsets_past_32_bits():
    m, n = 600001, 4096  # 2.4e9 values
    g = torch.Generator(device=DEV).manual_seed(1)
    X = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    rows = torch.randn(2048, n, generator=g, device=DEV).bfloat16()
    for i in range(0, m, 2048):
        X[i:i + 2048] = rows[:min(2048, m - i)]
    Y, mean, rstd = nv.svm_layer_norm(X, save=True)
    part = nv.svm_layer_norm(rows)
    last = (m - 1) // 2048 * 2048
    for i in (0, 524288, last):
        r = min(2048, m - i)
        assert torch.equal(Y[i:i + r], part[:r])
    del Y
    dY = torch.zeros_like(X)
    dY[-1] = 1.0
    dX, dw, db = nv.svm_layer_norm_backward(dY, X, mean, rstd)
    xh = (X[-1].double() - mean[-1].double()) * rstd[-1].double()
    close(dw, xh, 8 * E * (1 + xh.abs()), "bf16")
    assert bool((db == 1.0).all())
    assert not bool(dX[:-1].any())


# ------------------------------------------------------------------ hinge


def hinge64(S, lab, scale):
    S = S.double()
    m, n = S.shape
    want_lab = lab.long()
    seen = (want_lab >= 0) & (want_lab < max(n, 2))
    y = -torch.ones_like(S)
    if n == 1:
        y[want_lab == 1] = 1
    else:
        idx = torch.nonzero(seen)[:, 0]
        y[idx, want_lab[idx]] = 1
    gap = (1 - y * S).clamp(min=0) * seen[:, None]
    return scale * (gap ** 2).sum(), -2 * scale * y * gap, gap


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n", [(1, 1), (1, 2), (7, 3), (256, 1), (100, 10),
                                 (1000, 7), (33, 257), (5, 5000),
                                 (100000, 10), (70001, 3)])
def test_hinge(m, n, t):
    g = torch.Generator(device=DEV).manual_seed(m + 1000 * n)
    S = torch.randn(m, n, generator=g, device=DEV).to(TYPES[t])
    lab = torch.randint(-1, max(n, 2) + 1, (m,), generator=g, device=DEV,
                        dtype=torch.int32)
    loss, dS = nv.svm_hinge_loss(S, lab)
    want, grad, gap = hinge64(S, lab, 1 / m)
    # each square is good to 4 units; their sum is held in 64 bits
    assert abs(float(loss) - float(want)) <= 8 * E * float(want) + 1e-30
    close(dS, grad, 4 * E * (grad.abs() + 2 / m * E), t)
    l2, none = nv.svm_hinge_loss(S, lab, scale=0.5, need_grad=False)
    assert none is None
    assert abs(float(l2) - float(want) * m / 2) <= 8 * E * float(want) * m


def test_hinge_rows_left_out():
    S = torch.full((6, 3), float("nan"), device=DEV)
    lab = torch.tensor([-1, 3, -7, 100, -1, 5], dtype=torch.int32, device=DEV)
    loss, dS = nv.svm_hinge_loss(S, lab)
    assert float(loss) == 0.0 and not bool(dS.any())
    S[1] = torch.tensor([0.5, -2.0, 3.0])
    lab[1] = 2
    loss, dS = nv.svm_hinge_loss(S, lab, scale=1.0)
    assert float(loss) == 1.5 ** 2
    assert dS[1].tolist() == [3.0, 0.0, 0.0]
    assert not bool(dS[[0, 2, 3, 4, 5]].any())


def test_hinge_nan_score_of_a_labelled_row_is_seen():
    S = torch.zeros(4, 2, device=DEV)
    S[2, 1] = float("nan")
    lab = torch.zeros(4, dtype=torch.int32, device=DEV)
    loss, dS = nv.svm_hinge_loss(S, lab)
    assert math.isnan(float(loss))
    assert math.isnan(float(dS[2, 1])) and bool(torch.isfinite(dS[:2]).all())


def test_hinge_empty():
    S = torch.empty(0, 4, device=DEV)
    loss, dS = nv.svm_hinge_loss(S, torch.empty(0, dtype=torch.int32,
                                                device=DEV))
    assert float(loss) == 0.0 and dS.shape == (0, 4)


def test_hinge_strided():
    g = gen(41)
    B = rnd(g, 300, 12)
    lab = torch.randint(0, 5, (300,), generator=g).int().to(DEV)
    want, grad, _ = hinge64(B[:, 3:8], lab, 1 / 300)
    loss, dS = nv.svm_hinge_loss(B[:, 3:8], lab)
    assert abs(float(loss) - float(want)) <= 8 * E * float(want)
    close(dS, grad, 4 * E * grad.abs(), "f32")


def test_hinge_gradient_against_differences():
    g = gen(42)
    S = rnd(g, 30, 4)
    lab = torch.randint(0, 4, (30,), generator=g).int().to(DEV)
    _, dS = nv.svm_hinge_loss(S, lab)
    d = torch.randn(30, 4, generator=g).to(DEV).double()
    want = directional(lambda s: hinge64(s, lab, 1 / 30)[0], S.double(), d)
    have = float((dS.double() * d).sum())
    assert abs(have - want) <= 1e-5 * (1 + abs(want))


# ------------------------------------------------------------------ AdamW


HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05,
             grad_scale=0.7)


def held64(x, steps, signed):
    x = x.view(-1, 256)
    top = x.abs().amax(1, keepdim=True)
    top = torch.where(top > 1e-30, top, 0)
    y = (steps * (x.abs() / top).nan_to_num(0).sqrt())
    c = y.round()
    if not signed:
        c = torch.where((x > 0) & (top > 0), c.clamp(min=1), c)
    return (top * x.sign() * (c / steps) ** 2).view(-1)


def adam_tensors(t, gt, sizes, g):
    ps = [(torch.randn(*s, generator=g, device=DEV) * 0.1).to(TYPES[t])
          for s in sizes]
    return ps, lambda: [(torch.randn(*s, generator=g, device=DEV)
                         * 0.01).to(TYPES[gt]) for s in sizes]


SHAPES = [(1,), (3, 5), (256,), (257,), (0, 4), (16, 16), (1000, 33), (7,),
          (255, 3)]


@pytest.mark.parametrize("t,gt,master", [("f32", "f32", False),
                                         ("bf16", "bf16", True),
                                         ("bf16", "f32", True),
                                         ("bf16", "bf16", False),
                                         ("f16", "f16", True),
                                         ("f16", "f32", False)])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(t, gt, master, bits):
    g = torch.Generator(device=DEV).manual_seed(5)
    ps, grads = adam_tensors(t, gt, SHAPES * 8, g)  # several launches' worth
    at, total = nv.svm_adamw_parts(ps)
    st = list(nv.svm_adamw_states(ps, bits=bits, master=master))
    h = HYPER
    for step in range(1, 5):
        # the reference starts every step from the states the kernel holds
        if bits == 8:
            m0, v0 = (x.double() for x in nv.svm_adamw_state(*st[:4]))
        else:
            m0, v0 = st[0].double(), st[1].double()
        w0 = torch.zeros(total, dtype=torch.float64, device=DEV)
        for a, p in zip(at, ps):
            w0[a:a + p.numel()] = p.double().reshape(-1)
        if master:
            w0 = st[4].double().clone()
        gs = grads()
        gr = torch.zeros_like(w0)
        for a, x in zip(at, gs):
            gr[a:a + x.numel()] = x.double().reshape(-1)
        gr *= h["grad_scale"]
        nv.svm_adamw_step(ps, gs, *st, step=step, **h)
        m = h["beta1"] * m0 + (1 - h["beta1"]) * gr
        v = h["beta2"] * v0 + (1 - h["beta2"]) * gr ** 2
        up = (h["lr"] / (1 - h["beta1"] ** step) * m
              / (torch.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"]))
        p = w0 * (1 - h["lr"] * h["weight_decay"]) - up
        mabs = (h["beta1"] * m0).abs() + ((1 - h["beta1"]) * gr).abs()
        # some ten operations, each good to 2^-24 of its terms
        tol = 8 * E * (w0.abs() + up.abs()
                       + up.abs() * mabs / m.abs().clamp(min=1e-300))
        for a, x in zip(at, ps):
            n = x.numel()
            close(x.reshape(-1), p[a:a + n], tol[a:a + n], t)
        if master:
            close(st[4], p, tol, "f32")
            for a, x in zip(at, ps):
                n = x.numel()
                assert torch.equal(st[4][a:a + n].to(x.dtype),
                                   x.reshape(-1))
        tm, tv = 4 * E * mabs, 4 * E * v
        if bits == 32:
            close(st[0], m, tm, "f32")
            close(st[1], v, tv, "f32")
        else:
            hm, hv = nv.svm_adamw_state(*st[:4])
            # within half a step of the code: |d sqrt(x / top)| <= 1/2 steps
            for got, want, steps in ((hm.double(), m, 127),
                                     (hv.double().sqrt(), v.sqrt(), 254)):
                top = want.view(-1, 256).abs().amax(1, keepdim=True)
                q = lambda x: (x.view(-1, 256).abs()  # noqa: E731
                               / top.clamp(min=1e-300)).sqrt()
                least = 0.5 if steps == 127 else 1.0
                off = (q(got) - q(want)).abs() * steps
                small = q(want) * steps < 1
                assert bool((off <= torch.where(small, least, 0.5)
                             + 1e-3).all()), float(off.max())
                same = (got * want >= 0)
                assert bool(same.all())


def test_adamw_8_bit_codes_are_those_of_the_definition():
    # one step from zero states: the codes of the definition in 64 bits,
    # but for values within 2^-18 of a code's edge
    g = torch.Generator(device=DEV).manual_seed(9)
    p = torch.randn(4096, generator=g, device=DEV)
    x = torch.randn(4096, generator=g, device=DEV)
    st = nv.svm_adamw_states([p], bits=8)
    nv.svm_adamw_step([p], [x], *st, step=1)
    hm, hv = nv.svm_adamw_state(*st[:4])
    m = 0.1 * x.double()
    r = (0.001 * x.double() ** 2).sqrt()
    for got, want, steps, signed in ((hm.double(), m, 127, True),
                                     (hv.double().sqrt(), r, 254, False)):
        ref = held64(want, steps, signed)
        top = want.view(-1, 256).abs().amax(1, keepdim=True)
        edge = (want.view(-1, 256).abs() / top).sqrt() * steps
        near = ((edge % 1) - 0.5).abs().view(-1) < 2.0 ** -10
        ok = (got - ref).abs() <= 8 * E * ref.abs()
        assert bool((ok | near).all())
        assert int(near.sum()) < 64


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_second_moments_below_the_normal_range(bits):
    # v of some 1e-42 to 1e-40 is subnormal, its square root is not: codes
    # and steps as from that square root (of v as 32 bits hold it)
    g = torch.Generator().manual_seed(10)
    x = (3e-20 * 10 ** torch.rand(1024, generator=g)) \
        * torch.randn(1024, generator=g).sign()
    x[::7] = 0.0
    p = torch.zeros(1024, device=DEV)
    st = nv.svm_adamw_states([p], bits=bits)
    nv.svm_adamw_step([p], [x.to(DEV)], *st, lr=1.0, eps=0.0,
                      weight_decay=0.0, step=1)
    v = x * x * torch.tensor(1.0 - 0.999, dtype=torch.float32)
    assert float(v.max()) < 2.0 ** -126
    r = v.double().sqrt()
    live = x != 0
    want = -(0.1 * x.double() / 0.1) / (r / math.sqrt(1.0 - 0.999))
    off = (p.cpu().double() - want).abs()[live]
    assert bool((off <= 16 * E * want.abs()[live]).all())
    assert bool(p.cpu()[~live].isnan().all())  # 0 / 0: eps is 0
    if bits == 8:
        y = 254 * (r.view(-1, 256) / r.view(-1, 256).amax(1, keepdim=True)
                   ).sqrt().view(-1)
        near = ((y % 1) - 0.5).abs() < 2.0 ** -10
        code = st[1].cpu().double()
        assert bool((code == y.round())[~near].all())
        assert int(near.sum()) < 32


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_not_finite_and_zero_gradients(bits):
    p = torch.ones(600, device=DEV)
    q = p.clone()
    g = torch.full((600,), 0.01, device=DEV)
    st, s2 = (nv.svm_adamw_states([p], bits=bits) for _ in range(2))
    nv.svm_adamw_step([q], [g], *s2, step=1)
    bad = g.clone()
    bad[300] = float("nan")
    bad[301] = float("inf")
    nv.svm_adamw_step([p], [bad], *st, step=1)
    hit = torch.zeros(600, dtype=torch.bool, device=DEV)
    hit[300] = hit[301] = True
    # the others move as if those were not there
    assert torch.equal(p[~hit], q[~hit])
    assert math.isnan(float(p[300])) and math.isnan(float(p[301]))
    vals = [nv.svm_adamw_state(*s[:4]) if bits == 8 else s[:2]
            for s in (st, s2)]
    for a, b in zip(*vals):
        assert torch.equal(a[:600][~hit], b[:600][~hit])
        assert not bool(torch.isfinite(a[300:302]).any())
    # zero states and zero gradients: weight decay alone
    z = torch.ones(300, device=DEV)
    s3 = nv.svm_adamw_states([z], bits=bits)
    nv.svm_adamw_step([z], [torch.zeros(300, device=DEV)], *s3, step=1,
                      lr=0.1, weight_decay=0.5)
    assert torch.equal(z, torch.full_like(z, 0.95))


def test_adamw_8_bit_follows_32_bit():
    # a quadratic bowl: both kinds of states come down to it alike
    g = torch.Generator(device=DEV).manual_seed(2)
    goal = torch.randn(2000, generator=g, device=DEV)
    ends = []
    for bits in (32, 8):
        p = torch.zeros(2000, device=DEV)
        st = nv.svm_adamw_states([p], bits=bits)
        for step in range(1, 401):
            nv.svm_adamw_step([p], [p - goal], *st, step=step, lr=1e-2,
                              weight_decay=0.0)
        ends.append(float((p - goal).square().mean()))
    assert ends[0] < 1e-2 and ends[1] < 2e-2, ends


def test_adamw_odd_alignment():
    g = torch.Generator(device=DEV).manual_seed(4)
    base, gb = (torch.randn(3001, generator=g, device=DEV) for _ in range(2))
    for t in ("f32", "bf16"):
        p, x = base.to(TYPES[t])[1:2002], gb.to(TYPES[t])[3:2004]
        p2, x2 = p.clone(), x.clone()
        st, s2 = (nv.svm_adamw_states([p], bits=8) for _ in range(2))
        nv.svm_adamw_step([p], [x], *st, step=1)
        nv.svm_adamw_step([p2], [x2], *s2, step=1)
        assert torch.equal(p, p2)
        for a, b in zip(st[:4], s2[:4]):
            assert torch.equal(a, b)


# ------------------------------------------- streams, graphs, determinism


def _step(X, W, b, w, lab, ps, st, step=3):
    """A layer, a norm, the loss and the way back, and one update."""
    H, Z = nv.svm_linear(X, W, b, act="gelu", save=True)
    N, mean, rstd = nv.svm_layer_norm(H, w, save=True)
    loss, dN = nv.svm_hinge_loss(N, lab)
    dH, dw, _ = nv.svm_layer_norm_backward(dN, H, mean, rstd, w)
    dX, dW, db = nv.svm_linear_backward(dH, X, W, Z, act="gelu")
    nv.svm_adamw_step(ps, [dW, db, dw], *st, step=step)
    return loss, dX, dW, db, dw


def _setup(t, m=200, k=72, n=40):
    g = torch.Generator(device=DEV).manual_seed(77)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    X, W, b, w = (r(m, k).to(TYPES[t]), (r(n, k) * 0.1).to(TYPES[t]),
                  r(n).to(TYPES[t]), (1 + 0.1 * r(n)).to(TYPES[t]))
    lab = torch.randint(0, n, (m,), generator=g, device=DEV,
                        dtype=torch.int32)
    return X, W, b, w, lab


@pytest.mark.parametrize("t", list(TYPES))
def test_repeats_bit_for_bit_and_on_another_stream(t):
    X, W, b, w, lab = _setup(t)
    outs = []
    side = torch.cuda.Stream()
    for where in (None, None, side):
        ps = [W.clone(), b.clone(), w.clone()]
        st = nv.svm_adamw_states(ps, bits=8)
        torch.cuda.synchronize()
        if where is None:
            out = _step(X, *ps[:2], ps[2], lab, ps, st)
        else:
            with torch.cuda.stream(where):
                out = _step(X, *ps[:2], ps[2], lab, ps, st)
        torch.cuda.synchronize()
        outs.append([x.clone() for x in out] + ps + list(st[:4]))
    for other in outs[1:]:
        for a, c in zip(outs[0], other):
            assert torch.equal(a, c)
    # the stream of a call, with inputs that have to be copied first
    got = nv.svm_linear(X.t().contiguous().t(), W, b, act="gelu", stream=side)
    side.synchronize()
    assert torch.equal(got, nv.svm_linear(X, W, b, act="gelu"))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_captured_into_a_graph(t):
    X, W, b, w, lab = _setup(t)
    ps = [W, b, w]
    st = nv.svm_adamw_states(ps, bits=8)
    start = [x.clone() for x in ps + list(st[:4])]

    def restore():
        for x, s in zip(ps + list(st[:4]), start):
            x.copy_(s)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            _step(X, W, b, w, lab, ps, st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(X, W, b, w, lab, ps, st)
    for turn in range(4):
        X.add_(0.01)
        restore()
        torch.cuda.synchronize()
        want = [x.clone() for x in _step(X, W, b, w, lab, ps, st)]
        want += [x.clone() for x in ps + list(st[:4])]
        restore()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(list(outs) + ps + list(st[:4]), want):
            assert torch.equal(a, c), turn


def test_numpy_and_mixed_types_are_refused():
    X = torch.randn(4, 8, device=DEV)
    for call in (lambda: nv.svm_linear(np.zeros((4, 8), np.float32), X),
                 lambda: nv.svm_linear(X.cpu(), X),
                 lambda: nv.svm_linear(X, X.double()),
                 lambda: nv.svm_layer_norm(X.int()),
                 lambda: nv.svm_hinge_loss(X, torch.zeros(4, device=DEV))):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == nv.SVM_E_UNSUPPORTED
    for call in (lambda: nv.svm_linear(X, X.bfloat16()),
                 lambda: nv.svm_linear(X, X[:, :7].contiguous()),
                 lambda: nv.svm_linear(X, X, out=X[:, :4]),
                 lambda: nv.svm_linear(X, X, X[0]),
                 lambda: nv.svm_linear(X, X, act="swish"),
                 lambda: nv.svm_linear_backward(X[:, :4], X, X, None,
                                                act="gelu"),
                 lambda: nv.svm_hinge_loss(X, torch.zeros(
                     3, dtype=torch.int32, device=DEV)),
                 lambda: nv.svm_adamw_step([X], [X[:2]], X, X)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == nv.SVM_E_INVALID
