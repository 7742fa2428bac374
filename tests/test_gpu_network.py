"""The feature network with group norm, clipped steps and 4-bit weights: the
operators run together as a program uses them."""
import math

import numpy as np
import pytest
import torch

from paper_1706_05544_amd import native as nv
from paper_1706_05544_amd import workloads
from paper_1706_05544_amd.features import FeatureNet, PackedNet, patches

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_patches():
    X = torch.arange(2 * 36).view(2, 36)
    P = patches(X, 6, 3)
    assert P.shape == (2, 4, 9)
    img = X.view(2, 6, 6)
    assert torch.equal(P[1, 2], img[1, 3:, :3].reshape(-1))
    assert torch.equal(P[0, 1], img[0, :3, 3:].reshape(-1))


def reference(net, X, labels, groups):
    """Loss and gradients of the network in 64 bits, by torch's autograd on
    the CPU."""
    ps = [p.double().cpu().requires_grad_() for p in net.parameters]
    x, lab = X.double().cpu(), labels.long().cpu()
    it = iter(ps)
    nxt = lambda k: [next(it) for _ in range(k)]  # noqa: E731
    gelu = lambda z: 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))  # noqa: E731
    W, b = nxt(2)
    H = gelu(x @ W.t() + b)
    for _ in net.blocks:
        w, c, W, b = nxt(4)
        r = H.view(*H.shape[:2], groups, -1)
        d = r - r.mean((1, 3), keepdim=True)
        N = d / torch.sqrt((d * d).mean((1, 3), keepdim=True) + 1e-5)
        H = H + gelu(N.view(H.shape) * w + c) @ W.t() + b
    W, b = nxt(2)
    S = H.flatten(1) @ W.t() + b
    y = 2.0 * torch.nn.functional.one_hot(lab, S.shape[1]) - 1
    loss = (1 - y * S).clamp(min=0).square().sum() / len(lab)
    loss.backward()
    return float(loss.detach()), [p.grad for p in ps]


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4),
                                       (torch.bfloat16, 0.1),
                                       (torch.float16, 0.02)])
def test_gradients(dtype, tol):
    # tolerances: 32 bits some 12 layers deep of sums of 200 terms (1e-5 each
    # at the worst); 16 bits: each of some 12 stored tensors rounds its values
    # by up to u, 2^-8 or 2^-11, of which the norms of gradients keep a few
    net = FeatureNet(16, 48, 2, 5, dtype=dtype, seed=1, groups=6,
                     positions=9)
    for p in net.parameters:  # no zeros left among norms and biases
        p.add_(0.1 * torch.randn(p.shape, generator=torch.Generator()
                                 .manual_seed(p.numel())).to(DEV, dtype))
    g = torch.Generator().manual_seed(2)
    X = torch.randn(100, 9, 16, generator=g).to(DEV, dtype)
    labels = torch.randint(0, 5, (100,), generator=g).int().to(DEV)
    loss, S, grads = net.gradients(X, labels)
    assert torch.equal(S, net.scores(X))
    want, ref = reference(net, X, labels, 6)
    assert abs(float(loss) - want) <= tol * want
    for p, a, b in zip(net.parameters, grads, ref):
        assert a.shape == p.shape and a.dtype == p.dtype
        off = float((a.double().cpu() - b).norm() / b.norm())
        assert off <= tol, (tuple(p.shape), off)
    # the norm that a step clips by is that of these gradients
    norm, factor = nv.svm_grad_norm(grads, 0.5)
    exact = math.sqrt(sum(float(x.double().square().sum()) for x in grads))
    assert abs(float(norm) - exact) <= 2.0 ** -23 * exact
    assert abs(float(factor) * exact - 0.5) <= 2.0 ** -22


@pytest.mark.parametrize("groups", [0, 4])
@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32),
                                        (torch.bfloat16, 8)])
def test_clipped_training_and_serving(dtype, bits, groups):
    w = workloads.make("C4", n=4000, n_test=1000)
    cut = lambda A: patches(A, 28, 4) if groups else A  # noqa: E731
    X, Xt = (cut(torch.from_numpy(a).to(DEV, dtype)) for a in (w.X, w.Xt))
    labels = torch.from_numpy(w.y).to(DEV)
    net = FeatureNet(X.shape[-1], 32 if groups else 128, 2, w.n_classes,
                     dtype=dtype, bits=bits, groups=groups,
                     positions=X.shape[1] if groups else 1)
    for _ in range(3):
        for i in range(0, 4000, 250):
            net.step(X[i:i + 250], labels[i:i + 250], lr=2e-3, clip=1.0)
            assert net.norm.shape == ()
    hits = (net.scores(Xt).float().argmax(1).cpu().numpy() == w.yt).mean()
    assert hits > 0.9, hits
    # a batch with a NaN leaves everything as it was
    held = [t.clone() for t in net.parameters + [s for s in net.states
                                                 if s is not None]]
    bad = X[:250].clone()
    bad[3, 0] = math.nan
    net.step(bad, labels[:250], clip=1.0)
    assert not math.isfinite(float(net.norm))
    for a, b in zip(net.parameters + [s for s in net.states if s is not None],
                    held):
        assert torch.equal(a, b)
    # served: the layers on what 4 bits keep of the weights, one row and many
    served = net.packed(32)
    assert isinstance(served, PackedNet)
    plain = FeatureNet(X.shape[-1], 32 if groups else 128, 2, w.n_classes,
                       dtype=dtype, groups=groups,
                       positions=X.shape[1] if groups else 1)
    for p, q in zip(plain.parameters, net.parameters):
        p.copy_(q)
    for to, layer in zip([plain.first] + [b[2:] for b in plain.blocks]
                         + [plain.head],
                         [served.first] + [b[2:] for b in served.blocks]
                         + [served.head]):
        to[0].copy_(nv.svm_unpack_weights(layer[0]))
    # (sums in another order: some steps of the type through the layers)
    tol = 1e-4 if dtype == torch.float32 else 0.1
    for n in (1, 7, 1000):
        a, b = served.scores(Xt[:n]).double(), plain.scores(Xt[:n]).double()
        assert float((a - b).norm() / b.norm()) <= tol
    got = served.scores(Xt).float().argmax(1).cpu().numpy()
    assert float(np.mean(got == w.yt)) > 0.85


def test_a_clipped_step_captured_into_a_graph():
    g = torch.Generator().manual_seed(4)
    X = torch.randn(60, 9, 16, generator=g).to(DEV)
    labels = torch.randint(0, 5, (60,), generator=g).int().to(DEV)
    net = FeatureNet(16, 24, 1, 5, groups=4, positions=9)
    keep = net.parameters + [s for s in net.states if s is not None]
    start = [t.clone() for t in keep]

    def run():
        loss = net.step(X, labels, clip=0.1)
        net.steps -= 1
        return loss

    run()
    for t, s in zip(keep, start):
        t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = run()
    for turn in range(4):
        X.mul_(0.9)
        for t, s in zip(keep, start):
            t.copy_(s)
        eager = run().clone()
        want = [t.clone() for t in keep]
        for t, s in zip(keep, start):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, eager)
        for a, b in zip(keep, want):
            assert torch.equal(a, b), turn
