"""A network that is served in 4-bit weights stands by itself: training its
model on does not change it."""
import pytest
import torch

from paper_1706_05544_amd.features import FeatureNet

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("groups", [0, 4])
def test_training_on_leaves_the_served_network_as_it_is(groups):
    g = torch.Generator().manual_seed(3)
    X = torch.randn(40, *([9, 16] if groups else [16]), generator=g).to(DEV)
    y = torch.randint(0, 5, (40,), generator=g).int().to(DEV)
    net = FeatureNet(16, 24, 2, 5, groups=groups, positions=9)
    served = net.packed(32)
    before, own = served.scores(X), net.scores(X)
    for _ in range(3):
        net.step(X, y, lr=0.05)
    assert not torch.equal(net.scores(X), own)
    assert torch.equal(served.scores(X), before)
