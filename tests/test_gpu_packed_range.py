"""Layers on packed weights at inputs near the end of the range: what is
finite comes out finite, however many rows there are."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_packed import DEV, TYPES, gen, rnd

pytestmark = pytest.mark.gpu

E, U = 2.0 ** -23, {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 4, 5, 16, 40, 1030])
def test_sums_past_32_bits_before_their_scale(m, group, t):
    # codes of up to 6 and inputs of 2^125 make sums past 2^128, scales of
    # 2^-9 or so bring them back
    n, k = 70, 700
    g = gen(1000 * m + group)
    P = nv.svm_pack_weights(rnd(g, n, k, by=2.0 ** -8, t=t), group)
    W = nv.svm_unpack_weights(P).double()
    X = (1 + torch.rand(m, k, generator=g, device=DEV)).mul(2.0 ** 125).to(
        TYPES[t])
    X[0, 1::2] *= -1
    Y = nv.svm_linear_packed(X, P)
    want = X.double() @ W.t()
    assert bool(torch.isfinite(Y).all())
    # sums of k terms in 32 bits, in any order
    lim = k * E * (X.double().abs() @ W.abs().t()) + U[t] * want.abs()
    assert bool(((Y.double() - want).abs() <= lim * (1 + E)).all())


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_one_row_past_the_range_changes_no_other(t):
    g = gen(31)
    P = nv.svm_pack_weights(rnd(g, 70, 700, by=2.0 ** -8, t=t), 64)
    for m in (3, 16, 40):
        X = rnd(g, m, 700, t=t)
        clean = nv.svm_linear_packed(X, P)
        X[1] = 2.0 ** 126
        Y = nv.svm_linear_packed(X, P)
        assert bool(torch.isfinite(Y).all())
        keep = [i for i in range(m) if i != 1]
        off = (Y[keep].double() - clean[keep].double()).abs()
        lim = 700 * E * (X[keep].double().abs()
                         @ nv.svm_unpack_weights(P).double().abs().t())
        assert bool((off <= lim + 2 * U[t] * clean[keep].double().abs()).all())
