"""Weights in 4 bits and the linear layer on them, against their definitions.

The codes and scales are the definition's exactly (a division and comparisons
in 32 bits, correctly rounded on either side), and so is what they stand for.
The layer is then compared with 64 bits on those weights: K products of 32-bit
factors, summed in 32 bits, are off by at most about (K + 8) 2^-23 of the sum
of their magnitudes (a factor of X in three parts holds all its bits), the
activations are Lipschitz with at most 1.13 and good to a few units of
2^-24 (1 + z^2), and the result is rounded once, by half a step.
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
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rnd(g, *shape, by=1.0, t="f32"):
    return (torch.randn(shape, generator=g, device=DEV) * by).to(TYPES[t])


def held(W, group):
    """What 4 bits keep of W, on the CPU: the scales by their bits, the
    magnitudes by their distances in 64 bits."""
    t, (n, k) = W.dtype, W.shape
    pad = torch.nn.functional.pad(W.float().cpu(), (0, -k % group))
    pad = pad.view(n, -1, group)
    top = pad.abs().amax(2)
    bad = ~torch.isfinite(pad).all(2)
    sixth = torch.tensor(1.0) / torch.tensor(6.0)  # in 32 bits
    s = (torch.where(bad, 0, top) * sixth).view(torch.int32) >> 18 << 18
    s = s.view(torch.float32)
    if t == torch.float16:
        s = (s.double() * 2.0 ** 23).floor().float() * 2.0 ** -23
    x = (pad.abs() / s[..., None]).double().nan_to_num(0, 0, 0)
    off = (x[..., None] - GRID).abs()
    least = off.amin(-1, keepdim=True)
    near = off == least                    # two of them in the middle
    even = torch.tensor([1, 0, 1, 0, 1, 0, 1, 0], dtype=torch.bool)
    pick = near & (even | (near.sum(-1, keepdim=True) == 1))
    v = (pick * GRID).sum(-1) * s[..., None].double()
    v = torch.where(pad < 0, -v, v)
    v = torch.where(bad[..., None], math.nan, v)
    return v.reshape(n, -1)[:, :k], s


def same_values(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 1), (1, 31), (3, 33), (15, 127),
                                 (16, 128), (17, 129), (10, 784), (333, 501), (70, 4097)])
def test_pack_and_unpack(n, k, group, t):
    W = rnd(gen(n * k + group), n, k, by=k ** -0.5, t=t)
    P = nv.svm_pack_weights(W, group)
    assert P.shape == (n, k) and P.dtype == W.dtype
    got = nv.svm_unpack_weights(P)
    assert got.dtype == W.dtype and got.shape == W.shape
    assert same_values(got.cpu().double(), held(W, group)[0])
    # the largest magnitude of a group is held to within a sixth
    off = (got.double() - W.double()).abs()
    assert float(off.max()) <= float(W.double().abs().max()) / 6 * 1.04


@pytest.mark.parametrize("t", list(TYPES))
def test_pack_borders_and_ends_of_the_range(t):
    # every border between two magnitudes, and its neighbours
    s = 0.25
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]) * s
    W = torch.zeros(16, 64)
    eps = torch.finfo(TYPES[t]).eps
    W[0, :8], W[1, :8], W[2, :8] = mid, mid * (1 + eps), mid * (1 - eps)
    W[3:6] = -W[0:3]
    W[0:6, 8] = 6.0 * s                    # the scale
    fin = torch.finfo(TYPES[t])
    W[6, :3] = torch.tensor([fin.max, -fin.max / 2, fin.max / 12.5])
    W[7, :3] = torch.tensor([fin.tiny, fin.tiny / 2, -fin.tiny / 7])
    W[8, :4] = fin.smallest_normal * 0 + 2.0 ** (
        {"f32": -149, "bf16": -133, "f16": -24}[t]) * torch.tensor(
            [1.0, 2.0, 13.0, 60.0])
    W[9, 0] = -0.0
    W[10, 5], W[10, 40] = math.nan, 2.0
    W[11, 5], W[11, 40] = math.inf, 2.0
    W[12, 5], W[12, 40] = -math.inf, 2.0
    # a sixth of it falls just short of six bits, and its product with the
    # 32-bit number nearest to 1/6 on them
    W[13, 0], W[13, 1] = 0.11132811754941940, 0.05
    W = W.to(TYPES[t]).to(DEV)
    for group in (32, 64):
        P = nv.svm_pack_weights(W, group)
        got = nv.svm_unpack_weights(P).cpu().double()
        want = held(W, group)[0]
        assert same_values(got, want)
        assert got[10:13, :32].isnan().all()
        if t == "f32":
            assert float(got[13, 0]) == 6 * 0.0185546875
        if group == 32:  # the next group is untouched
            assert got[10:13, 40].eq(2.0).logical_or(
                (got[10:13, 40] - 2.0).abs() < 0.07).all()


@pytest.mark.parametrize("t", list(TYPES))
def test_pack_strided(t):
    g = gen(5)
    B = rnd(g, 40, 300, t=t)
    for W in (B[:, 3:203], B[::2, :77], B.t(), B[:, ::3]):
        a = nv.svm_pack_weights(W, 32)
        b = nv.svm_pack_weights(W.contiguous(), 32)
        assert torch.equal(a.data, b.data)


def act64(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return {"tanh": torch.tanh, "cos": torch.cos}.get(name, lambda x: x)(z)


def check(X, P, b, R, act, t, W=None, **kw):
    Y = nv.svm_linear_packed(X, P, b, R, act=act, **kw)
    W = nv.svm_unpack_weights(P) if W is None else W
    x, w = X.double().reshape(-1, X.shape[-1]), W.double()
    z, mag = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    y = act64(act, z)
    tol = 1.13 * (X.shape[-1] + 8) * E * mag + 4 * E * (1 + z * z)
    if R is not None:
        r = R.double().reshape(y.shape)
        y, tol = y + r, tol + E * (y.abs() + r.abs())
    got = Y.double().reshape(y.shape)
    lim = tol * (1 + U[t]) + U[t] * y.abs() * (1 + 1e-6) + FLOOR[t]
    assert bool(((got - y).abs() <= lim).all()), float(
        ((got - y).abs() / lim).max())
    return Y


# rows on both sides of every kernel's limits, outputs round a tile of 16,
# inputs round a step of 32 and a chunk of 128
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m", [1, 2, 4, 5, 16, 17, 32, 33, 48, 64, 65, 129,
                               300])
def test_rows(m, t):
    for n, k, group in ((40, 784, 32), (333, 501, 64), (17, 4097, 128),
                        (1, 1, 32), (1030, 33, 64)):
        g = gen(m * 7 + n)
        X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
        b, R = rnd(g, n, t=t), rnd(g, m, n, t=t)
        P = nv.svm_pack_weights(W, group)
        check(X, P, b, R, "gelu", t)
        check(X, P, None, None, "none", t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("k", [1, 7, 8, 31, 32, 33, 64, 100, 127, 128, 129,
                               255, 256, 1000, 1024, 1025, 2049, 20000])
def test_inputs(k, t):
    g = gen(k)
    n = 50
    W = rnd(g, n, k, by=k ** -0.5, t=t)
    for group in (32, 128):
        P = nv.svm_pack_weights(W, group)
        for m in (1, 3, 20):
            check(rnd(g, m, k, t=t), P, rnd(g, n, t=t), None, "silu", t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "tanh",
                                 "cos"])
@pytest.mark.parametrize("m", [2, 30, 100])
def test_acts(m, act, t):
    g = gen(m)
    X, W = rnd(g, m, 100, t=t), rnd(g, 72, 100, by=0.2, t=t)
    b, R = rnd(g, 72, t=t), rnd(g, m, 72, t=t)
    P = nv.svm_pack_weights(W, 32)
    check(X, P, b, R, act, t)
    check(X, P, b, None, act, t)
    check(X, P, None, R, act, t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", [(1, 4096, 16384), (3, 16384, 1000),
                                   (32, 4096, 4096), (64, 2048, 6000),
                                   (2000, 784, 2048)])
def test_large(m, k, n, t):
    g = gen(m + k)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
    b, R = rnd(g, n, t=t), rnd(g, m, n, t=t)
    check(X, nv.svm_pack_weights(W, 64), b, R, "gelu", t)


# both sides of where rows count as many, odd sizes, every number of tiles to
# a block; many rows in 32 bits take three products for six
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k,n", [(1024, 100, 90), (1025, 100, 90),
                                   (1100, 33, 17), (384, 1030, 1040),
                                   (385, 1030, 1040), (500, 2052, 700),
                                   (2, 130, 8200), (16, 130, 8200),
                                   (16, 130, 16500), (33, 130, 2800)])
def test_many_rows_and_many_tiles(m, k, n, t):
    g = gen(m + n)
    X, W = rnd(g, m, k, t=t), rnd(g, n, k, by=k ** -0.5, t=t)
    b, R = rnd(g, n, t=t), rnd(g, m, n, t=t)
    for group in (32, 128):
        check(X, nv.svm_pack_weights(W, group), b, R, "gelu", t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m", [3, 24, 50, 90, 1030])
def test_strides_in_place_and_nothing_beside(m, t):
    g = gen(m + 1)
    k, n = 100, 90
    P = nv.svm_pack_weights(rnd(g, n, k, by=0.1, t=t), 32)
    for shift in (0, 1, 3, 8):
        X = rnd(g, m, k + 29, t=t)[:, shift:shift + k]
        R = rnd(g, m, n + 13, t=t)[:, shift:shift + n]
        b = rnd(g, 2 * n, t=t)[::2]
        out = torch.full((m + 2, n + 11), 7.0, dtype=TYPES[t], device=DEV)
        o = out[1:-1, shift:shift + n]
        check(X, P, b, R, "tanh", t, out=o)
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[1:-1, shift:shift + n] = False
        assert bool((out[rest] == 7.0).all())
        want = o.clone()
        o.copy_(R)
        nv.svm_linear_packed(X, P, b, o, act="tanh", out=o)
        assert torch.equal(o, want)
    # a transposed input, leading dimensions, one row without any
    X = rnd(g, k, m, t=t).t()
    Y = check(X, P, None, None, "none", t)
    Y3 = nv.svm_linear_packed(X.reshape(1, m, 1, k), P)
    assert Y3.shape == (1, m, 1, n) and torch.equal(Y3.view(m, n), Y)
    assert nv.svm_linear_packed(X[0].contiguous(), P).shape == (n,)


@pytest.mark.parametrize("t", list(TYPES))
def test_rows_do_not_depend_on_each_other(t):
    # an infinity or NaN in a row stays there, and shows; no rows are allowed
    g = gen(11)
    P = nv.svm_pack_weights(rnd(g, 60, 200, by=0.1, t=t), 32)
    W = nv.svm_unpack_weights(P).double()
    for m in (4, 16, 40, 1040):
        X = rnd(g, m, 200, t=t)
        clean = nv.svm_linear_packed(X, P)
        bad = X.clone()
        bad[1, 199], bad[2, 5] = math.nan, math.inf
        got = nv.svm_linear_packed(bad, P)
        keep = [i for i in range(m) if i not in (1, 2)]
        assert torch.equal(got[keep], clean[keep])
        assert bool(got[1].isnan().all())
        # the sign of the weight times infinity, NaN where the weight is 0
        w = W[:, 5]
        assert bool((got[2].double() == w * math.inf)[w != 0].all())
        assert bool(got[2][w == 0].isnan().all())
    assert nv.svm_linear_packed(X[:0], P).shape == (0, 60)


def test_a_group_that_is_not_a_number_shows_in_its_output_alone():
    g = gen(12)
    W = rnd(g, 40, 100)
    W[7, 50] = math.nan
    P = nv.svm_pack_weights(W, 32)
    for m in (1, 10, 100):
        Y = nv.svm_linear_packed(rnd(g, m, 100), P)
        assert bool(Y[:, 7].isnan().all())
        assert not bool(Y[:, :7].isnan().any() or Y[:, 8:].isnan().any())


def test_32_bit_inputs_keep_all_their_bits():
    # weights of 6 and 0 (scale 1): six times the input, whose three parts of
    # eight bits hold it exactly from 2^-109 on; two additions in 32 bits, each
    # off by 2^-23
    k = 64
    W = torch.zeros(k, 128, device=DEV)
    W[:, :64].fill_diagonal_(6.0)
    P = nv.svm_pack_weights(W, 64)
    g = gen(13)
    for m in (1, 16, 33, 1030):
        x = torch.randn(m, 128, generator=g, device=DEV)
        x[:, 64:] = 0.0
        for by in (1.0, 2.0 ** -100, 2.0 ** 115):
            Y = nv.svm_linear_packed(x * by, P).double()
            want = x[:, :64].double() * by * 6.0
            # (the third part of x below 2^-109 falls under bf16's smallest
            # step, 2^-133, and is cut by less than that: six times it here)
            lim = 2 * E * want.abs() + 6 * 2.0 ** -133
            assert bool(((Y - want).abs() <= lim).all())


def test_streams_and_replays():
    g = gen(14)
    W, R = rnd(g, 300, 260, t="bf16"), rnd(g, 300, 1090, t="bf16").t()
    P = nv.svm_pack_weights(W, 64)
    X = {m: rnd(g, 260, m, t="bf16").t() for m in (2, 30, 1090)}
    side = torch.cuda.Stream()
    for m, x in X.items():
        want = nv.svm_linear_packed(x, P, None, R[:m], act="gelu")
        Q = nv.svm_pack_weights(W, 64, stream=side)
        got = nv.svm_linear_packed(x, Q, None, R[:m], act="gelu", stream=side)
        back = nv.svm_unpack_weights(Q, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(Q.data, P.data)
        assert torch.equal(back, nv.svm_unpack_weights(P))
        torch.cuda.synchronize()
        xc = x.contiguous()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = nv.svm_linear_packed(xc, P, None, R[:m], act="gelu")
        for turn in range(4):
            xc.mul_(0.9)
            eager = nv.svm_linear_packed(xc, P, None, R[:m], act="gelu")
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager), turn


def test_offsets_past_32_bits():
    # 2.4e9 bytes of codes, 4.8e9 weights: the first, a middle and the last
    # rows against weights of their own
    n, k = 40000, 120000
    g = gen(15)
    rows = rnd(g, 500, k, by=k ** -0.5, t="bf16")
    W = torch.empty(n, k, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 500):
        W[i:i + 500] = rows
    P = nv.svm_pack_weights(W, 128)
    assert P.data.numel() > 1 << 31
    part = nv.svm_pack_weights(rows, 128)
    w = nv.svm_unpack_weights(part)
    for m in (1, 20):
        X = rnd(g, m, k, t="bf16")
        Y = nv.svm_linear_packed(X, P)
        want = nv.svm_linear_packed(X, part)
        assert torch.equal(Y, want.repeat(1, n // 500))
    W.zero_()
    back = nv.svm_unpack_weights(P)
    for i in (0, 20000, n - 500):
        assert torch.equal(back[i:i + 500], w)


def test_packed_weights_are_made_again_from_their_bytes():
    g = gen(16)
    P = nv.svm_pack_weights(rnd(g, 50, 70), 32)
    Q = nv.PackedWeights(P.data.cpu().to(DEV), [50, 70], 32, torch.float32)
    X = rnd(g, 3, 70)
    assert torch.equal(nv.svm_linear_packed(X, P), nv.svm_linear_packed(X, Q))
    short = nv.PackedWeights(P.data[:-16], P.shape, 32, torch.float32)
    for call, code in (
            (lambda: nv.svm_linear_packed(X, short), nv.SVM_E_INVALID),
            (lambda: nv.svm_unpack_weights(short), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X.half(), P), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X[:, :69], P), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X, X), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X, nv.PackedWeights(
                P.data.cpu(), P.shape, 32, torch.float32)), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X, nv.PackedWeights(
                P.data, P.shape, 48, torch.float32)), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X, nv.PackedWeights(
                P.data, P.shape, 32, torch.float64)), nv.SVM_E_INVALID),
            (lambda: nv.PackedWeights(P.data[::2], P.shape, 32, torch.float32),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_pack_weights(X, 48), nv.SVM_E_INVALID),
            (lambda: nv.svm_pack_weights(X.cpu()), nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_linear_packed(X, P, act="swish"), nv.SVM_E_INVALID),
            (lambda: nv.svm_linear_packed(X, P, out=torch.empty(
                3, 49, device=DEV)), nv.SVM_E_INVALID)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == code
