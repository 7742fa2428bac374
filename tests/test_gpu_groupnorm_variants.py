"""Group norm and its gradients against 64 bits in every variant of their
kernels that a call can reach: threads and pieces of a slab, groups of whole
eights of channels and others, whole samples and chunks.  test_group_plan.py
asks the plan which variant each size takes, and that none is missing."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_groupnorm import DEV, EPS, TYPES, Ref, check, gen, rnd

pytestmark = pytest.mark.gpu

SIZES = [(14677, 22, 1, 1), (744, 315, 2, 1), (3596, 77, 2, 2),
         (1, 8, 73416, 69), (826, 835, 1, 1), (6, 22, 8480, 4),
         (1, 42, 27400, 25), (2, 5, 116788, 28), (8207, 18, 8, 1),
         (346, 72, 80, 5), (1, 2094, 2, 2), (1, 174, 96, 1),
         (6, 44537, 1, 1), (512, 1045, 2, 1), (2, 33, 34848, 33),
         (1082, 2, 384, 16), (1, 2097, 10, 5), (1, 2063, 16, 2),
         (5, 5, 124944, 114), (3, 371, 4098, 1), (2, 523, 4368, 2),
         # larger and odder ones of the same
         (229, 619, 120, 30), (67, 666, 504, 7), (1253, 18, 125, 5),
         (991, 69, 60, 15), (6, 4042, 768, 24), (13, 7871, 64, 2)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,p,c,groups", SIZES)
def test_every_variant(n, p, c, groups, t):
    g = gen(n, p, c, groups)
    X = (rnd(g, n, p, c, by=1.5) + rnd(g, n, 1, 1) + rnd(g, c)).to(TYPES[t])
    w, b = (1 + rnd(g, c, by=0.2)).to(TYPES[t]), rnd(g, c, by=0.3, t=t)
    dY, R = rnd(g, n, p, c, t=t), rnd(g, n, p, c, t=t)
    check(X, groups, w, b, "gelu", t, R, dY)


def test_the_last_samples_of_2_6e9_values():
    n, p, c, groups = 5000, 1024, 512, 32
    g = gen(16)
    X = torch.empty(n, p, c, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 50):
        X[i:i + 50] = rnd(g, 50, p, c, t="bf16") + i / n
    w, b = rnd(g, c, t="bf16"), rnd(g, c, t="bf16")
    Y, mean, rstd = nv.svm_group_norm(X, groups, w, b, eps=EPS, act="silu",
                                      save=True)
    for i in (0, 2499, n - 1):
        Ref(X[i:i + 1], groups, w, b, "silu").forward(
            Y[i:i + 1], mean[i:i + 1], rstd[i:i + 1], "bf16")
