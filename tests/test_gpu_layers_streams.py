"""The feature-map calls on another stream than torch's current one: what the
binding copies first has to be there when the call's work begins."""
import pytest
import torch

from paper_1706_05544_amd import native as nv

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m", [24, 700])  # few rows, and tiles
def test_copies_of_inputs_are_waited_for(t, m):
    k, n = 96, 136
    g = torch.Generator(device=DEV).manual_seed(m)
    r = lambda *s: torch.randn(  # noqa: E731
        *s, generator=g, device=DEV).to(TYPES[t])
    X, W, b, R = r(k, m).t(), r(k, n).t(), r(2 * n)[::2], r(n, m).t()
    want = nv.svm_linear(X, W, b, R, act="gelu", save=True)
    back = nv.svm_linear_backward(R, X, W, want[1], act="gelu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    for _ in range(20):  # torch's stream has work in front of the copies
        busy = (busy @ busy).clamp(-1, 1)
    got = nv.svm_linear(X, W, b, R, act="gelu", save=True, stream=side)
    # (torch's stream may run ahead: its later calls wait for nothing here)
    grads = nv.svm_linear_backward(R, X, W, want[1], act="gelu", stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, c in zip(got + grads, want + back):
        assert torch.equal(a, c)
