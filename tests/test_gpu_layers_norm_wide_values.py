"""Gradients of layer norm at rows of large values: what lies past a row's end
in its lanes adds nothing, at any width."""
import pytest
import torch

from paper_1706_05544_amd import native as nv
from test_gpu_layers import DEV, E, TYPES, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 127, 128, 501, 1000, 2047, 4095, 8191,
                               12001, 16383, 20001])
def test_constant_rows_of_large_values(n, t):
    # xh = 0 in the row, and mean rstd = 6.3e38 past its end
    m, eps = 7, 1e-5
    X = torch.full((m, n), 2e36, device=DEV).to(TYPES[t])
    g = torch.Generator(device=DEV).manual_seed(n)
    X[3] = torch.randn(n, generator=g, device=DEV).to(TYPES[t])
    dY = torch.randn(m, n, generator=g, device=DEV).to(TYPES[t])
    x = X.double()
    mean = x.mean(1).float()
    rstd = (1 / (x.var(1, unbiased=False) + eps).sqrt()).float()
    got = nv.svm_layer_norm_backward(dY, X, mean, rstd)
    rs = rstd.double()[:, None]
    dy = dY.double()
    rows = [i for i in range(m) if i != 3]
    want = rs * (dy - dy.mean(1, keepdim=True))
    tol = rs * E * (4 * dy.abs() + (n / 64 + 20)
                    * dy.abs().mean(1, keepdim=True))
    close(got[0][rows], want[rows], tol[rows], t)
    assert bool(torch.isfinite(got[0]).all())
    assert bool(torch.isfinite(got[1]).all())
