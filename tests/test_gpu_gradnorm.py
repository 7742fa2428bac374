"""The norm of all gradients, its clipping factor and the AdamW step that
takes it, against their definitions in 64 bits.

Squares are exact in 64 bits (24 + 24 bits) and their sum is good to N 2^-53
of itself, so norm and factor are off by the rounding to 32 bits, 2^-24, and
next to nothing besides: 2^-23 is allowed.
"""
import math

import pytest
import torch

from paper_1706_05544_amd import native as nv

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E = 2.0 ** -23
INF = float("inf")


def norm64(gs, scale=1.0):
    return abs(scale) * math.sqrt(sum(float(g.double().square().sum())
                                      for g in gs))


def check(gs, most, scale=1.0, **kw):
    norm, factor = nv.svm_grad_norm(gs, most, grad_scale=scale, **kw)
    assert norm.shape == () and norm.dtype == torch.float32
    want = norm64(gs, scale)
    assert abs(float(norm) - want) <= E * want
    f = most / want if want > most else 1.0
    assert abs(float(factor) - f) <= E * f
    return norm, factor


# round a unit of 4096 values, a turn of the blocks (2048 units) and a launch
# of 128 tensors
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("sizes", [
    [1], [7], [4095], [4096], [4097], [0, 5, 0], [255, 256, 257, 2047, 2049],
    [4096 * 2048 + 3], [1000] * 300, [3] * 129, [10000000, 1, 12345]])
def test_norm_and_factor(sizes, t):
    g = torch.Generator(device=DEV).manual_seed(sum(sizes))
    gs = [torch.randn(n, generator=g, device=DEV).to(TYPES[t]) for n in sizes]
    want = norm64(gs)
    check(gs, 0.25 * want)
    check(gs, 4.0 * want)
    check(gs, 1.0, -0.125)
    _, f = check(gs, INF)
    assert float(f) == 1.0
    _, f = nv.svm_grad_norm(gs, 0.0)
    assert float(f) == 0.0


def test_types_mixed_and_shapes_as_they_come():
    g = torch.Generator(device=DEV).manual_seed(3)
    gs = [torch.randn(s, generator=g, device=DEV).to(TYPES[t])
          for s, t in (((33, 65), "f32"), ((129,), "bf16"), ((), "f16"),
                       ((2, 3, 5), "bf16"), ((0, 4), "f32"))]
    gs.append(torch.randn(40, 30, generator=g, device=DEV).t())
    gs.append(torch.randn(9000, generator=g, device=DEV)[1::2])
    gs.append(torch.randn(5001, generator=g, device=DEV).half()[3:])
    gs.append(torch.randn(7, 1, generator=g, device=DEV).expand(7, 9))
    check(gs, 1.0)


def test_ends_of_the_range():
    # squares past 32 bits, above and below; a norm past 32 bits
    big = torch.full((1000,), 3e38, device=DEV)
    norm, factor = nv.svm_grad_norm([big], 1.0)
    assert float(norm) == INF and not math.isnan(float(factor))
    want = 1.0 / (3e38 * math.sqrt(1000))  # (subnormal: steps of 2^-149)
    assert abs(float(factor) - want) <= want * E + 2.0 ** -149
    check([big], 1.0, 1e-30)
    check([torch.full((1000,), 1e19, device=DEV)], 1e3)
    check([torch.full((100,), 1e-40, device=DEV)], 1e-41)
    check([torch.full((100,), 6e-8, device=DEV, dtype=torch.float16)], 1e-9)
    check([torch.full((70000,), 65504.0, device=DEV, dtype=torch.float16)], 1)
    zero = torch.zeros(500, device=DEV)
    for most in (0.0, 1.0, INF):
        norm, factor = nv.svm_grad_norm([zero], most)
        assert float(norm) == 0.0 and float(factor) == 1.0


@pytest.mark.parametrize("bad", [float("nan"), INF, -INF])
@pytest.mark.parametrize("t", list(TYPES))
def test_gradients_that_are_not_finite(t, bad):
    gs = [torch.ones(5000, device=DEV, dtype=TYPES[t]) for _ in range(3)]
    gs[1][4999] = bad
    norm, factor = nv.svm_grad_norm(gs, 1.0)
    assert not math.isfinite(float(norm)) and math.isnan(float(factor))
    _, factor = nv.svm_grad_norm(gs, INF)
    assert math.isnan(float(factor))


SHAPES = [(1,), (3, 5), (256,), (257,), (0, 4), (1000, 33), (255, 3)]
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05,
             step=3)


def _tensors(t, gt, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda s, by, to: (torch.randn(s, generator=g, device=DEV)  # noqa
                           * by).to(TYPES[to])
    return [r(s, 0.1, t) for s in SHAPES], [r(s, 0.01, gt) for s in SHAPES]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("t,gt,master", [("f32", "f32", False),
                                         ("bf16", "bf16", True),
                                         ("bf16", "f32", False),
                                         ("f16", "f16", True),
                                         ("f16", "f16", False)])
def test_a_clipped_step_is_the_step_of_the_scaled_gradients(t, gt, master,
                                                            bits):
    # (grad_scale factor in 32 bits is what the plain step takes as its
    # grad_scale: the same bits)
    ps, gs = _tensors(t, gt, 5)
    qs = [p.clone() for p in ps]
    a, b = (nv.svm_adamw_states(x, bits=bits, master=master)
            for x in (ps, qs))
    norm, factor = nv.svm_grad_norm(gs, 0.3, grad_scale=0.5)
    assert 0 < float(factor) < 1
    for _ in range(3):
        nv.svm_adamw_step(ps, gs, *a, grad_scale=0.5, factor=factor, **HYPER)
        nv.svm_adamw_step(qs, gs, *b, grad_scale=float(0.5 * factor), **HYPER)
    for x, y in zip(ps + list(a), qs + list(b)):
        assert (x is None and y is None) or torch.equal(x, y)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_of_gradients_that_are_not_finite_is_left_out(bits):
    ps, gs = _tensors("bf16", "bf16", 6)
    st = nv.svm_adamw_states(ps, bits=bits, master=True)
    nv.svm_adamw_step(ps, gs, *st, **HYPER)
    before = [x.clone() for x in ps + [s for s in st if s is not None]]
    gs[3][100] = float("nan")
    norm, factor = nv.svm_grad_norm(gs, 1.0)
    nv.svm_adamw_step(ps, gs, *st, factor=factor, **HYPER)
    for f in (INF, -INF):
        nv.svm_adamw_step(ps, gs, *st, factor=torch.full((), f, device=DEV),
                          **HYPER)
    for x, y in zip(ps + [s for s in st if s is not None], before):
        assert torch.equal(x, y)


def test_the_clipped_step_moves_as_its_definition_in_64_bits():
    # from zero states at step 1, eps 0: m / sqrt(v) is the sign, whatever the
    # factor; with eps the factor shows
    g = torch.Generator(device=DEV).manual_seed(8)
    p = torch.randn(2500, generator=g, device=DEV)
    x = torch.randn(2500, generator=g, device=DEV)
    norm, factor = nv.svm_grad_norm([x], 1e-3)
    q = p.clone()
    st = nv.svm_adamw_states([q])
    nv.svm_adamw_step([q], [x], *st, lr=0.1, eps=1e-4, weight_decay=0.0,
                      step=1, factor=factor)
    c = x.double() * (1e-3 / x.double().norm())
    want = p.double() - 0.1 * c / (c.abs() + 1e-4)
    # some ten operations, each good to a unit of 2^-23 of its terms
    assert bool(((q.double() - want).abs()
                 <= 16 * E * (p.double().abs() + 0.1)).all())
    assert bool(((st[0][:2500].double() - 0.1 * c).abs() <= 4 * E * c.abs()).all())


def test_another_stream_and_repeated_replays():
    g = torch.Generator(device=DEV).manual_seed(9)
    base = torch.randn(300, 400, generator=g, device=DEV)
    ps = [torch.randn(400, 300, generator=g, device=DEV)]
    st = nv.svm_adamw_states(ps)
    start = [x.clone() for x in [ps[0], st[0], st[1]]]

    def step(stream=None):
        # (a gradient whose rows have to be copied first)
        norm, factor = nv.svm_grad_norm([base.t()], 0.5, stream=stream)
        nv.svm_adamw_step(ps, [base.t()], *st, factor=factor, step=2,
                          stream=stream)
        return norm, factor

    def restore():
        for x, s in zip([ps[0], st[0], st[1]], start):
            x.copy_(s)

    def held():
        return [x.clone() for x in (ps[0], st[0], st[1])]

    out = step()
    want = [x.clone() for x in out] + held()
    restore()
    side = torch.cuda.Stream()
    out = step(side)
    side.synchronize()
    for a, b in zip(list(out) + held(), want):
        assert torch.equal(a, b)
    restore()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(4):
        base.mul_(1.5)
        restore()
        want = [x.clone() for x in step()] + held()
        restore()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(list(out) + held(), want):
            assert torch.equal(a, b), turn


def test_refusals():
    g = torch.ones(4, device=DEV)
    for call, code in (
            (lambda: nv.svm_grad_norm([]), nv.SVM_E_INVALID),
            (lambda: nv.svm_grad_norm([g, g.cpu()]), nv.SVM_E_INVALID),
            (lambda: nv.svm_grad_norm([g, None]), nv.SVM_E_INVALID),
            (lambda: nv.svm_grad_norm([g.cpu()]), nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_grad_norm([g.double()]), nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_grad_norm([g], -1.0), nv.SVM_E_INVALID),
            (lambda: nv.svm_grad_norm([g], float("nan")), nv.SVM_E_INVALID),
            (lambda: nv.svm_grad_norm([g], 1.0, grad_scale=INF),
             nv.SVM_E_INVALID),
            (lambda: nv.svm_adamw_step([g], [g.clone()],
                                       *nv.svm_adamw_states([g]), factor=0.5),
             nv.SVM_E_UNSUPPORTED),
            (lambda: nv.svm_adamw_step(
                [g], [g.clone()], *nv.svm_adamw_states([g]),
                factor=torch.ones(2, device=DEV)), nv.SVM_E_INVALID)):
        with pytest.raises(nv.SvmError) as e:
            call()
        assert e.value.status == code
