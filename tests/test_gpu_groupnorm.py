"""Group norm with an activation and its gradients against their definitions
in 64 bits.

Tolerances, with E = 2^-23 and n values to a group.  The mean: sums of n terms
in 32 bits, in parts of at most some thousand each, are off by at most
L E of the mean magnitude A of the values, L = 64 + n / 256 covering the
longest chain of additions (8 columns, the positions of a thread, the rows of a
block, the groups' columns).  The squared deviations of the rounded mean add
its error squared.  rstd is good to L E of itself then, plus the share that
the mean's error has in the variance.  An output is off by the error of
x - mean times rstd and weight, a few units of its terms, and 1.13 times that
after the activation (their largest slope).  A gradient dX is made of terms
a, mean(a) and xh mean(a xh), each off by a few units and L E of the mean
magnitudes; the slopes of the activations are good to a few units of
(1 + z^2) and change by at most 1.13 of z's error.  relu's slope is settled
exactly.  Each result is rounded once, by half a step of its type.
"""
import math

import pytest
import torch

from paper_1706_05544_amd import native as nv

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
FLOOR = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
E = 2.0 ** -23
EPS = 1e-5
ACTS = ("none", "relu", "gelu", "silu", "tanh", "cos")


def gen(*key):
    return torch.Generator(device=DEV).manual_seed(
        sum(k * 10007 ** i for i, k in enumerate(key)) % (1 << 31))


def rnd(g, *shape, by=1.0, t="f32"):
    return (torch.randn(shape, generator=g, device=DEV) * by).to(TYPES[t])


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


def close(got, want, tol, t):
    lim = tol * (1 + U[t]) + U[t] * want.abs() * (1 + 1e-6) + FLOOR[t]
    off = (got.double() - want).abs()
    assert got.shape == want.shape
    assert bool((off <= lim).all()), float((off / lim).max())


class Ref:
    """The operator in 64 bits on X viewed as samples x positions x channels,
    with its tolerances."""

    def __init__(self, X, groups, w, b, act):
        self.shape = X.shape
        n, c = X.shape[0], X.shape[-1]
        self.x = X.double().reshape(n, -1, c)
        self.p, self.c, self.g = self.x.shape[1], c, groups
        one = torch.ones(c, dtype=torch.float64, device=DEV)
        self.w = one if w is None else w.double()
        self.b = 0 * one if b is None else b.double()
        self.act = act
        self.size = self.p * c // groups
        self.L = 64 + self.size / 256

    def rows(self, x):
        n = x.shape[0]
        return x.view(n, self.p, self.g, -1).transpose(1, 2).reshape(
            n, self.g, -1)

    def wide(self, s):
        """A value of each sample and group, at each of their elements."""
        return s.repeat_interleave(self.c // self.g, 1)[:, None, :]

    def forward(self, Y, mean, rstd, t):
        r = self.rows(self.x)
        mu = r.mean(2)
        var = (r - mu[..., None]).square().mean(2)
        rs = 1 / torch.sqrt(var + EPS)
        tm = self.L * E * r.abs().mean(2)
        if mean is not None:
            assert mean.shape == mu.shape and rstd.shape == mu.shape
            close(mean, mu, tm, "f32")
            ts = rs * (self.L * E + (tm * rs) ** 2)
            close(rstd, rs, ts, "f32")
        off = self.x - self.wide(mu)
        xh = off * self.wide(rs)
        z = xh * self.w + self.b
        txh = (self.wide(tm * rs) + 4 * E * xh.abs() + xh.abs() * self.wide(
            self.L * E + (tm * rs) ** 2))
        tz = txh * self.w.abs() + 2 * E * (z.abs() + self.b.abs())
        y, _ = act64(self.act, z)
        close(Y, y.view(self.shape), (1.13 * tz + 4 * E * (1 + z * z)).view(
            self.shape), t)

    def backward(self, got, dY, mean, rstd, res, t, need=(True,) * 3):
        mu, rs = mean.double(), rstd.double()
        off = self.x - self.wide(mu)
        xh = off * self.wide(rs)
        z = xh * self.w + self.b
        dy = dY.double().reshape(self.x.shape)
        _, slope = act64(self.act, z)
        tz = 4 * E * (xh * self.w).abs() + 2 * E * (z.abs() + self.b.abs())
        tslope = 0 if self.act in ("none", "relu") else (
            1.13 * tz + 6 * E * (1 + z * z))
        dz, tdz = dy * slope, dy.abs() * (tslope + E * slope.abs())
        a, ta = dz * self.w, (tdz + E * dz.abs()) * self.w.abs()
        m1 = self.rows(a).mean(2)
        m2 = self.rows(a * xh).mean(2)
        t1 = self.rows(ta + self.L * E * a.abs()).mean(2)
        t2 = self.rows((ta + (self.L + 4) * E * a.abs()) * xh.abs()).mean(2)
        dx = self.wide(rs) * (a - self.wide(m1) - xh * self.wide(m2))
        tdx = self.wide(rs) * (ta + self.wide(t1) + xh.abs() * self.wide(t2)
                               + 8 * E * (a.abs() + self.wide(m1.abs())
                                          + (xh * self.wide(m2)).abs()))
        if res is not None:
            r = res.double().reshape(self.x.shape)
            dx, tdx = dx + r, tdx + E * (dx.abs() + r.abs())
        m = self.x.shape[0] * self.p
        # columns: chains of the rows' sums, in a block and over the blocks
        long = (64 + m / 16) * E
        want = ((dx.view(self.shape), tdx.view(self.shape)),
                ((dz * xh).sum((0, 1)),
                 ((tdz + (long + 4 * E) * dz.abs()) * xh.abs()).sum((0, 1))),
                (dz.sum((0, 1)), (tdz + long * dz.abs()).sum((0, 1))))
        for x, (v, tol), asked in zip(got, want, need):
            assert (x is not None) == asked
            if asked:
                close(x, v, tol, t)


def check(X, groups, w, b, act, t, res=None, dY=None, back=True):
    ref = Ref(X, groups, w, b, act)
    Y, mean, rstd = nv.svm_group_norm(X, groups, w, b, eps=EPS, act=act,
                                      save=True)
    ref.forward(Y, mean, rstd, t)
    assert torch.equal(nv.svm_group_norm(X, groups, w, b, eps=EPS, act=act),
                       Y)
    if back:
        got = nv.svm_group_norm_backward(dY, X, groups, mean, rstd, w, b,
                                         act=act, residual=res)
        ref.backward(got, dY, mean, rstd, res, t)
    return Y, mean, rstd


# samples x positions x channels, groups: widths of a group that are no
# multiple of 8, one channel to a group, one group in all, a position or a
# sample alone, slabs of every size and the cut into chunks
SIZES = [(1, 1, 1, 1), (1, 1, 8, 8), (3, 1, 7, 7), (5, 1, 64, 8),
         (1, 49, 64, 8), (2, 9, 33, 11), (7, 5, 24, 3), (300, 1, 256, 8),
         (1000, 1, 40, 5), (33, 2, 1000, 4), (4, 196, 512, 32),
         (64, 196, 96, 6), (2, 3977, 231, 33), (1, 5000, 16, 16),
         (1, 70000, 8, 1), (1, 3000, 320, 1), (6, 1024, 130, 2),
         (2, 100, 4096, 1), (3, 7, 9000, 2), (1, 1, 50000, 1),
         (2, 33, 16384, 4), (1, 1, 131072, 64), (17, 64, 40, 1),
         (40, 300, 65, 13), (1, 300, 1, 1), (3, 900, 3, 1), (2, 90, 5, 5),
         (1, 40000, 7, 7)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,p,c,groups", SIZES)
def test_group_norm_and_gradients(n, p, c, groups, t):
    g = gen(n, p, c, groups)
    X = (rnd(g, n, p, c, by=1.5) + rnd(g, n, 1, 1) + rnd(g, c)).to(TYPES[t])
    w, b = (1 + rnd(g, c, by=0.2)).to(TYPES[t]), rnd(g, c, by=0.3, t=t)
    dY, R = rnd(g, n, p, c, t=t), rnd(g, n, p, c, t=t)
    check(X, groups, w, b, "silu", t, R, dY)
    check(X, groups, None, None, "none", t, None, dY)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n,p,c,groups", [(5, 30, 48, 6), (2, 4000, 35, 5)])
def test_acts(n, p, c, groups, act, t):
    g = gen(n, c)
    X, dY = rnd(g, n, p, c, by=2.0, t=t), rnd(g, n, p, c, t=t)
    w, b = (1 + rnd(g, c, by=0.2)).to(TYPES[t]), rnd(g, c, by=0.3, t=t)
    w[0], b[0] = 0.0, 0.0  # (z is 0 there: relu's slope at 0 is 0)
    check(X, groups, w, b, act, t, None, dY)
    check(X, groups, w, None, act, t, dY, dY)
    check(X, groups, None, b, act, t, None, dY)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,p,c,groups", [(64, 196, 512, 32),
                                          (4096, 1, 2048, 32),
                                          (2, 64 * 64, 640, 32),
                                          (3000, 49, 64, 8),
                                          (20000, 3, 30, 3)])
def test_large(n, p, c, groups, t):
    g = gen(n, p, 1)
    X, dY, R = (rnd(g, n, p, c, by=y, t=t) for y in (2.0, 1.0, 1.0))
    w, b = (1 + rnd(g, c, by=0.2)).to(TYPES[t]), rnd(g, c, by=0.3, t=t)
    check(X, groups, w, b, "gelu", t, R, dY)


@pytest.mark.parametrize("n,p,c,groups", [(4, 10, 24, 3), (1, 3000, 100, 4)])
def test_a_level_far_above_the_spread(n, p, c, groups):
    # deviations of 1 about 3000: the variance of the deviations, not a
    # difference of squares
    g = gen(n, p, 2)
    X = rnd(g, n, p, c) + 3000.0
    Y, mean, rstd = nv.svm_group_norm(X, groups, save=True)
    Ref(X, groups, None, None, "none").forward(Y, mean, rstd, "f32")
    assert bool(((rstd - 1).abs() < 0.2).all())


@pytest.mark.parametrize("act", ["none", "gelu", "silu", "tanh", "cos"])
def test_gradient_against_differences(act):
    n, p, c, groups = 3, 5, 12, 4
    g = gen(3, 5)
    X, dY = rnd(g, n, p, c), rnd(g, n, p, c)
    w, b = 1 + rnd(g, c, by=0.3), rnd(g, c, by=0.3)
    _, mean, rstd = nv.svm_group_norm(X, groups, w, b, act=act, save=True)
    grads = nv.svm_group_norm_backward(dY, X, groups, mean, rstd, w, b,
                                       act=act)

    def loss(x=X.double(), w=w.double(), b=b.double()):
        r = x.view(n, p, groups, -1)
        d = r - r.mean((1, 3), keepdim=True)
        xh = d / torch.sqrt(d.square().mean((1, 3), keepdim=True) + EPS)
        return (dY.double() * act64(act, xh.view(n, p, c) * w + b)[0]).sum()

    for name, v, got in zip("xwb", (X, w, b), grads):
        d = torch.randn(v.shape, generator=g, device=DEV).double()
        h = 1e-5
        want = float((loss(**{name: v.double() + h * d}) -
                      loss(**{name: v.double() - h * d})) / (2 * h))
        have = float((got.double() * d).sum())
        lim = float((got.double().abs() * d.abs()).sum()) * 200 * E + 1e-6
        assert abs(have - want) <= lim, (name, have, want)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,p,c,groups", [(6, 20, 36, 3), (2, 3000, 44, 4)])
def test_what_is_asked_for_and_in_place(n, p, c, groups, t):
    g = gen(n, 9)
    X, dY, R = (rnd(g, n, p, c, t=t) for _ in range(3))
    w, b = rnd(g, c, t=t), rnd(g, c, t=t)
    Y, mean, rstd = nv.svm_group_norm(X, groups, w, b, act="silu", save=True)
    inp = X.clone()
    assert nv.svm_group_norm(inp, groups, w, b, act="silu", out=inp) is inp
    assert torch.equal(inp, Y)
    full = nv.svm_group_norm_backward(dY, X, groups, mean, rstd, w, b,
                                      act="silu", residual=R)
    for need in ((True, False, False), (False, True, False),
                 (False, False, True), (False, True, True),
                 (True, True, False), (False, False, False)):
        got = nv.svm_group_norm_backward(dY, X, groups, mean, rstd, w, b,
                                         act="silu", residual=R, need=need)
        for a, f, asked in zip(got, full, need):
            assert (a is not None) == asked
            assert a is None or torch.equal(a, f)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,p,c,groups", [(4, 20, 36, 3), (2, 3000, 44, 4)])
def test_strides_and_nothing_beside(n, p, c, groups, t):
    g = gen(n, 11)
    for shift in (0, 1, 3, 8):
        X = rnd(g, n, p, c + 13, t=t)[..., shift:shift + c]
        dY = rnd(g, n, p, c + 9, t=t)[..., shift:shift + c]
        R = rnd(g, n, p, c + 21, t=t)[..., shift:shift + c]
        w, b = rnd(g, 2 * c, t=t)[::2], rnd(g, c + 1, t=t)[1:]
        Y, mean, rstd = check(X, groups, w, b, "tanh", t, R, dY)
        out = torch.full((n, p, c + 10), 7.0, dtype=TYPES[t], device=DEV)
        nv.svm_group_norm(X, groups, w, b, act="tanh",
                          out=out[..., shift:shift + c])
        assert torch.equal(out[..., shift:shift + c], Y)
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[..., shift:shift + c] = False
        assert bool((out[rest] == 7.0).all())
    # channels first, as it may come: copied
    X = rnd(g, n, c, p, t=t).transpose(1, 2)
    assert torch.equal(nv.svm_group_norm(X, groups),
                       nv.svm_group_norm(X.contiguous(), groups))


def test_dimensions():
    g = gen(1, 12)
    X = rnd(g, 3, 4, 5, 24)
    Y, mean, rstd = nv.svm_group_norm(X, 6, save=True)
    assert Y.shape == X.shape and mean.shape == (3, 6) == rstd.shape
    assert torch.equal(Y.view(3, 20, 24),
                       nv.svm_group_norm(X.view(3, 20, 24), 6))
    # no positions between: a row is a sample
    Z = nv.svm_group_norm(X.view(60, 24), 6)
    assert torch.equal(Z.view(60, 1, 24),
                       nv.svm_group_norm(X.view(60, 1, 24), 6))
    # one group over a row is layer norm, up to the order of the sums
    L = nv.svm_layer_norm(X.view(60, 24))
    assert float((nv.svm_group_norm(X.view(60, 24), 1) - L).abs().max()) < \
        1e-5
    # empty
    for shape in ((0, 5, 24), (0, 24), (3, 0, 24)):
        e = torch.empty(shape, device=DEV)
        Y, mean, rstd = nv.svm_group_norm(e, 6, save=True)
        assert Y.shape == shape and mean.shape == (shape[0], 6)
        dX, dw, db = nv.svm_group_norm_backward(e, e, 6, mean, rstd)
        assert dX.shape == shape
        assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("p", [6, 5000])
def test_what_is_not_finite_stays_in_its_group(p, t):
    g = gen(p, 13)
    X, dY = rnd(g, 3, p, 20, t=t), rnd(g, 3, p, 20, t=t)
    clean, mean, rstd = nv.svm_group_norm(X, 4, act="silu", save=True)
    back = nv.svm_group_norm_backward(dY, X, 4, mean, rstd, act="silu")
    for bad in (math.nan, math.inf):
        Z = X.clone()
        Z[1, p - 1, 7] = bad
        Y, m2, r2 = nv.svm_group_norm(Z, 4, act="silu", save=True)
        hit = torch.zeros_like(X, dtype=torch.bool)
        hit[1, :, 5:10] = True
        assert torch.equal(Y[~hit], clean[~hit])
        assert bool(Y[hit].isnan().all())
        G = dY.clone()
        G[1, 0, 7] = bad
        dX, dw, db = nv.svm_group_norm_backward(G, X, 4, mean, rstd,
                                                act="silu")
        assert torch.equal(dX[~hit], back[0][~hit])
        assert not bool(dX[hit].isfinite().any())
        keep = [c for c in range(20) if c != 7]
        assert torch.equal(dw[keep], back[1][keep])
        assert torch.equal(db[keep], back[2][keep])
        assert not math.isfinite(float(dw[7]) + float(db[7]))


def test_relu_slopes_at_the_border():
    # z within 32 bits' rounding of 0 on either side: the sign of the exact
    # value decides
    n, p, c = 2, 400, 16
    g = gen(14)
    X, dY = rnd(g, n, p, c), torch.ones(n, p, c, device=DEV)
    _, mean, rstd = nv.svm_group_norm(X, 2, save=True)
    w = torch.ones(c, device=DEV)
    wide = lambda s: s.double().repeat_interleave(8, 1)[:, None]  # noqa: E731
    xh = (X.double() - wide(mean)) * wide(rstd)
    # biases that put one position of each channel next to 0
    b = -xh[0, 3].float()
    z = xh + b.double()
    assert float(z[0, 3].abs().max()) < 1e-6
    _, _, db = nv.svm_group_norm_backward(dY, X, 2, mean, rstd, w, b,
                                          act="relu")
    assert torch.equal(db.double(), (z > 0).double().sum((0, 1)))


def test_streams_and_replays():
    for n, p, c, groups in ((5, 30, 48, 6), (2, 4000, 64, 4)):
        g = gen(n, 15)
        X = rnd(g, n, c, p, t="bf16").transpose(1, 2)
        dY, w, b = (rnd(g, n, p, c, t="bf16"), rnd(g, 2 * c, t="bf16")[::2],
                    rnd(g, c, t="bf16"))

        def both(x, stream=None):
            Y, mean, rstd = nv.svm_group_norm(x, groups, w, b, act="gelu",
                                              save=True, stream=stream)
            if stream is not None:
                torch.cuda.current_stream().wait_stream(stream)
            return (Y, mean, rstd) + nv.svm_group_norm_backward(
                dY, x, groups, mean, rstd, w, b, act="gelu", residual=dY,
                stream=stream)

        want = both(X)
        side = torch.cuda.Stream()
        got = both(X, side)
        side.synchronize()
        for a, c2 in zip(got, want):
            assert torch.equal(a, c2)
        torch.cuda.synchronize()
        xc = X.contiguous()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(xc)
        for turn in range(4):
            xc.mul_(1.1)
            eager = both(xc)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, c2 in zip(out, eager):
                assert torch.equal(a, c2), turn


def test_offsets_past_32_bits():
    # 2.6e9 values: the last samples against a call on them alone
    n, p, c, groups = 5000, 1024, 512, 32
    g = gen(16)
    rows = rnd(g, 50, p, c, t="bf16")
    X = torch.empty(n, p, c, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 50):
        X[i:i + 50] = rows
    Y, mean, rstd = nv.svm_group_norm(X, groups, act="silu", save=True)
    part = nv.svm_group_norm(rows, groups, act="silu")
    # (another cut of the rows may be taken for fewer samples: the sums'
    # order, within a step of the type)
    for i in (0, 2500, n - 50):
        off = (Y[i:i + 50].float() - part.float()).abs()
        assert bool((off <= part.float().abs() * 2 ** -7 + 1e-5).all())
    dY = torch.zeros_like(X)
    dY[-1] = rows[0]
    del Y
    dX, dw, db = nv.svm_group_norm_backward(dY, X, groups, mean, rstd,
                                            act="silu")
    ref = Ref(X[-1:], groups, None, None, "silu")
    ref.backward((dX[-1:], dw, db), dY[-1:], mean[-1:], rstd[-1:], None,
                 "bf16")
    assert not bool(dX[:-1].any())


def test_refusals():
    X = torch.randn(4, 6, 24, device=DEV)
    st = torch.zeros(4, 6, device=DEV)
    for call, code in (
            (lambda: nv.svm_group_norm(X, 5), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 0), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, -2, save=True), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X[0, 0], 2), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, X[0, 0, :23]), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, X[0, 0].half()),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, eps=-1.0), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, act="swish"), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, out=X[:, :3]), nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X, 6, out=X[..., :23]),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm(X.cpu(), 6), nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_group_norm(X.double(), 6), nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_group_norm_backward(X, X, 5, st, st),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm_backward(X, X[:, :3], 6, st, st),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm_backward(X, X, 6, st[:3], st),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_group_norm_backward(X, X, 6, st, st.half()),
             nv.SVM_E_UNSUPPORTED)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == code
