"""Steps that are left out because their gradients are not finite: the steps
after them are those of a training that never saw them."""
import math

import pytest
import torch

from paper_1706_05544_amd import native as nv
from paper_1706_05544_amd.features import FeatureNet

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E = 2.0 ** -23


def batches(n, dtype):
    g = torch.Generator().manual_seed(21)
    return [(torch.randn(40, 9, 16, generator=g).to(DEV, dtype),
             torch.randint(0, 5, (40,), generator=g).int().to(DEV))
            for _ in range(n)]


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32),
                                        (torch.bfloat16, 8)])
@pytest.mark.parametrize("bad_at", [(0,), (0, 1, 2), (1, 3), (4,)])
def test_training_goes_on_as_if_they_had_not_been(bad_at, dtype, bits):
    # (the corrections of a step after them come from powers of two numbers
    # in 64 bits on the device, on the host otherwise: the same in 32 bits but
    # where their last bits of 64 fall on either side of a border)
    make = lambda: FeatureNet(16, 24, 1, 5, dtype=dtype, bits=bits,  # noqa
                              groups=4, positions=9)
    a, b = make(), make()
    good = batches(5, dtype)
    for i, (X, y) in enumerate(good):
        if i in bad_at:
            bad = X.clone()
            bad[3, 0, 0] = math.nan
            a.step(bad, y, clip=0.1)
            assert not math.isfinite(float(a.norm))
        a.step(X, y, clip=0.1)
        b.step(X, y, clip=0.1)
        for p, q in zip(a.parameters + list(a.states),
                        b.parameters + list(b.states)):
            assert (p is None and q is None) or torch.equal(p, q), i
    # and without a clipping limit
    X, y = good[0]
    a.step(X, y)
    b.step(X, y)
    for p, q in zip(a.parameters, b.parameters):
        assert torch.equal(p, q)


KINDS = [("f32", "f32", False), ("bf16", "bf16", True), ("f16", "f32", False)]
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05)


def tensors(t, gt, sizes=(1, 15, 256, 257, 0, 33000)):
    g = torch.Generator(device=DEV).manual_seed(22)
    r = lambda n, to: torch.randn(n, generator=g, device=DEV).to(  # noqa
        TYPES[to])
    return [r(n, t) for n in sizes], [r(n, gt) for n in sizes]


def count():
    return torch.zeros((), dtype=torch.int64, device=DEV)


def nan():
    return torch.full((), math.nan, device=DEV)


def everything(ps, st):
    return ps + [s for s in st if s is not None]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("t,gt,master", KINDS)
def test_the_step_is_that_of_the_steps_taken(t, gt, master, bits):
    ps, gs = tensors(t, gt)
    qs = [p.clone() for p in ps]
    a, b = (nv.svm_adamw_states(x, bits=bits, master=master)
            for x in (ps, qs))
    c, taken = count(), 0
    _, f = nv.svm_grad_norm(gs, 0.5)
    for step, bad in enumerate((True, False, False, True, True, False), 1):
        # (the last without a factor: the count holds for it too)
        factor = nan() if bad else f if step < 6 else None
        nv.svm_adamw_step(ps, gs, *a, factor=factor, step=step, left_out=c,
                          **HYPER)
        if not bad:
            taken += 1
            nv.svm_adamw_step(qs, gs, *b, factor=factor, step=taken, **HYPER)
        assert int(c) == step - taken
        for x, y in zip(everything(ps, a), everything(qs, b)):
            assert torch.equal(x, y), step


def test_a_step_of_several_launches_counts_once():
    # more tensors than travel in one launch, and of several types
    ps, gs = [], []
    for t in TYPES:
        p, g = tensors(t, t, [7] * 60)
        ps, gs = ps + p, gs + g
    st = nv.svm_adamw_states(ps)
    c, before = count(), [p.clone() for p in ps]
    for k in range(1, 4):
        nv.svm_adamw_step(ps, gs, *st, factor=nan(), left_out=c, step=k)
        assert int(c) == k
    for p, q in zip(ps, before):
        assert torch.equal(p, q)


def test_a_count_past_the_step_is_the_first_step():
    for held in (3, 100, 2 ** 62):
        ps, gs = tensors("f32", "f32")
        qs = [p.clone() for p in ps]
        a, b = nv.svm_adamw_states(ps), nv.svm_adamw_states(qs)
        nv.svm_adamw_step(ps, gs, *a, step=3, left_out=count() + held)
        nv.svm_adamw_step(qs, gs, *b, step=1)
        for x, y in zip(ps, qs):
            assert torch.equal(x, y)


def test_far_steps():
    # corrections of far steps, as 64 bits on the host make them: within a
    # unit of 32 bits' last place
    for held, step in ((1, 2), (7, 1000), (500, 100000), (10, 10 ** 9)):
        ps, gs = tensors("f32", "f32", [5000])
        qs = [p.clone() for p in ps]
        a, b = nv.svm_adamw_states(ps), nv.svm_adamw_states(qs)
        kw = dict(lr=0.1, beta1=0.9, beta2=0.999, weight_decay=0.0)
        nv.svm_adamw_step(ps, gs, *a, step=step, left_out=count() + held, **kw)
        nv.svm_adamw_step(qs, gs, *b, step=step - held, **kw)
        # (rate and root each off by a rounding, the weight by another)
        moved = (ps[0].double() - qs[0].double()).abs()
        size = (qs[0].double() - tensors("f32", "f32", [5000])[0][0]).abs()
        assert bool((moved <= 4 * E * (size + qs[0].double().abs())).all())


def test_another_stream_and_replays():
    ps, gs = tensors("f32", "f32")
    st, c = nv.svm_adamw_states(ps), count()
    f = torch.ones((), device=DEV)
    keep = everything(ps, st) + [c]
    start = [x.clone() for x in keep]

    def run(stream=None):
        nv.svm_adamw_step(ps, gs, *st, factor=f, step=4, left_out=c,
                          stream=stream)

    def restore():
        for x, s in zip(keep, start):
            x.copy_(s)

    side = torch.cuda.Stream()
    for value in (1.0, math.inf, 0.5):
        f.fill_(value)
        restore()
        run()
        want = [x.clone() for x in keep]
        restore()
        run(side)
        side.synchronize()
        for x, y in zip(keep, want):
            assert torch.equal(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    restore()
    both = []
    for turn in (0, 1):  # eager, then replayed
        restore()
        for value in (math.nan, 1.0, math.nan, -math.inf, 0.25, 2.0):
            f.fill_(value)
            graph.replay() if turn else run()
            torch.cuda.synchronize()
        both.append([x.clone() for x in keep])
    assert int(both[1][-1]) == 3
    for x, y in zip(*both):
        assert torch.equal(x, y)
