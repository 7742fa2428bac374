"""Gradients of group norm at groups of large values: a block's slabs that
have no unit of their own add nothing, whatever the last sample's statistics."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_groupnorm import EPS, TYPES, Ref, gen, rnd

pytestmark = pytest.mark.gpu


# slabs of 8, 16 and 64 threads (32, 16 and 4 to a block), units that leave
# some of a block's free, groups of 8 channels and of other widths
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("n,p,c,groups", [
    (5, 1, 64, 8), (3, 1, 7, 7), (1000, 1, 64, 8), (1, 1, 8, 8),
    (5, 2, 64, 8), (1001, 3, 64, 8), (7, 5, 24, 3), (1001, 9, 64, 8),
    (301, 1, 256, 8), (5, 9, 33, 3), (1000, 1, 40, 5), (33, 2, 90, 3)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_a_last_sample_of_large_constants(n, p, c, groups, act, t):
    # its xh are 0 and its rstd 316; (1 - mean) rstd is -6e38
    g = gen(n, p, c)
    X, dY, R = (rnd(g, n, p, c, t=t) for _ in range(3))
    X[-1] = 2e36
    w, b = (1 + rnd(g, c, by=0.2)).to(TYPES[t]), rnd(g, c, by=0.3, t=t)
    r = X.double().reshape(n, p, groups, -1).transpose(1, 2).reshape(
        n, groups, -1)
    mean = r.mean(2).float()
    rstd = (1 / (r.var(2, unbiased=False) + EPS).sqrt()).float()
    assert bool((rstd[-1] > 316).all())
    got = nv.svm_group_norm_backward(dY, X, groups, mean, rstd, w, b, act=act,
                                     residual=R)
    for x in got:
        assert bool(torch.isfinite(x).all())
    Ref(X, groups, w, b, act).backward(got, dY, mean, rstd, R, t)
