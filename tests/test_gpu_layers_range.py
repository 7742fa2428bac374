"""32-bit products at both ends of the 32-bit range (values are held in three
bf16 parts, whose largest is 3.39e38 and whose smallest step is 2^-133).
Tolerances as in test_gpu_layers.py."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_layers import DEV, close, linear64

pytestmark = pytest.mark.gpu

# few rows, tiles of whole steps, tiles with a step that is not whole
SHAPES = [(9, 64, 66), (70, 64, 66), (300, 77, 130)]


def top(g, *shape):
    """Magnitudes in [3.38e38, 3.396e38): the largest that round to a bf16."""
    v = 3.38e38 + 1.59e36 * torch.rand(*shape, generator=g,
                                       dtype=torch.float64)
    sign = torch.randint(0, 2, shape, generator=g) * 2 - 1
    return (v * sign).float().to(DEV)


@pytest.mark.parametrize("m,k,n", SHAPES)
def test_factors_just_below_the_largest(m, k, n):
    g = torch.Generator().manual_seed(m)
    W = (torch.randn(n, k, generator=g) * 2.0 ** -90).to(DEV)
    X = top(g, m, k)
    y, _, _, tz = linear64(X, W, None, None, "none")
    close(nv.svm_linear(X, W), y, tz, "f32")
    y, _, _, tz = linear64(W, X, None, None, "none")
    close(nv.svm_linear(W, X), y, tz, "f32")
    # and across the summed index, as the gradients read them
    G = (torch.randn(m, n, generator=g) * 2.0 ** -90).to(DEV)
    dW = nv.svm_linear_backward(G, X, W, need=(False, True, False))[1]
    y, _, _, tz = linear64(G.t(), X.t(), None, None, "none")
    close(dW, y, tz, "f32")


@pytest.mark.parametrize("m,k,n", SHAPES)
@pytest.mark.parametrize("a", [-109, -118, -125, -130])
def test_small_factors_with_large_ones(m, k, n, a):
    # from 2^-109 on the three parts hold all 24 bits; below, a value is off
    # by at most half a bf16's smallest step, 2^-134
    g = torch.Generator().manual_seed(m)
    X = (torch.randn(m, k, generator=g) * 2.0 ** a).to(DEV)
    W = (torch.randn(n, k, generator=g) * 2.0 ** 100).to(DEV)
    y, _, _, tz = linear64(X, W, None, None, "none")
    lost = 2.0 ** -134 * W.double().abs().sum(1)
    close(nv.svm_linear(X, W), y, tz + lost, "f32")
    y, _, _, tz = linear64(W, X, None, None, "none")
    close(nv.svm_linear(W, X), y, tz + lost[:, None], "f32")


def test_smallest_values_that_are_held_whole():
    # magnitudes of at least 2^-109, products with 2^100: to 32 bits
    g = torch.Generator().manual_seed(3)
    v = (1 + torch.rand(80, 64, generator=g)) * 2.0 ** -109
    X = (v * (torch.randint(0, 2, v.shape, generator=g) * 2 - 1)).to(DEV)
    W = (torch.randn(70, 64, generator=g) * 2.0 ** 100).to(DEV)
    y, _, _, tz = linear64(X, W, None, None, "none")
    close(nv.svm_linear(X, W), y, tz, "f32")
