"""Operators around a feature network's training step and its serving, as
measurable cases.

A case is a dict of plain values.  Its ``kind`` says which operator one pass
goes through:

  grad_norm     the norm of all gradients of a network as one vector, and the
                factor that brings it down to a limit
  clipped_step  the same, and the AdamW step that takes the factor
  group_norm    group norm over samples x positions x channels, channels
                last, with an activation
  group_bwd     its gradients, the sums over all rows for weight and bias too
  linear4       Y = act(X W^T + b) + R with W in 4 bits, a scale to each group
                of inputs: the layer of a network that is served

Inputs are drawn on the GPU from the seed alone.  With ``own`` false a pass
computes the operator from elementary torch operations in 32 bits (long sums
of squares in 64), rounded once at the end; with ``own`` true it calls the
library.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu", "tanh")
EPS = 1e-5                      # group norm
ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
            step=100)
BLOCK = 256                     # states come in whole blocks of as many
# the magnitudes that 3 bits stand for, and the borders between them; a value
# on a border takes the even code
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def listed():
    return [
        # the gradients of a small network: launches are all there is
        dict(name="grad_norm_128_256x4_f32", kind="grad_norm", d=128,
             width=256, blocks=4, classes=10, type="f32", max_norm=1.0,
             grad_scale=1.0),
        # of a large one in 16 bits, scaled by a loss scale of 1024
        dict(name="grad_norm_784_4096x4_bf16", kind="grad_norm", d=784,
             width=4096, blocks=4, classes=10, type="bf16", max_norm=1.0,
             grad_scale=2.0 ** -10),
        # a training step of a small network with its norm clipped
        dict(name="clipped_step_128_256x4_f32", kind="clipped_step", d=128,
             width=256, blocks=4, classes=10, type="f32", max_norm=0.5,
             grad_scale=1.0, master=False),
        # of a large one, 16-bit weights with 32-bit masters
        dict(name="clipped_step_784_2048x6_bf16", kind="clipped_step", d=784,
             width=2048, blocks=6, classes=10, type="bf16", max_norm=1.0,
             grad_scale=0.25, master=True),
        # one image of 28 x 28 in patches of 4 x 4, a request of a serving
        # loop
        dict(name="group_norm_1x49x64_f32", kind="group_norm", samples=1,
             positions=49, channels=64, groups=8, type="f32", act="silu"),
        # a training batch of patches in a wide layer; the largest of its
        # kind
        dict(name="group_norm_512x196x512_bf16", kind="group_norm",
             samples=512, positions=196, channels=512, groups=32,
             type="bf16", act="silu"),
        # its gradients, with what goes past the norm
        dict(name="group_bwd_256x196x512_bf16", kind="group_bwd",
             samples=256, positions=196, channels=512, groups=32,
             type="bf16", act="silu", residual=True),
        # few large maps, odd in every size: groups of 7 channels, rows
        # without alignment
        dict(name="group_bwd_6x3977x231_f16",
             kind="group_bwd", samples=6, positions=3977, channels=231,
             groups=33, type="f16", act="gelu", residual=False),
        # one request through a layer: a row of 784 pixels
        dict(name="linear4_1x784x1024_bf16", kind="linear4", m=1, k=784,
             n=1024, group=32, type="bf16", act="gelu", residual=False),
        # one row through a wide residual layer
        dict(name="linear4_1x4096x16384_f16", kind="linear4", m=1, k=4096,
             n=16384, group=64, type="f16", act="silu", residual=True),
        # requests gathered into a batch
        dict(name="linear4_32x4096x4096_bf16", kind="linear4", m=32, k=4096,
             n=4096, group=64, type="bf16", act="gelu", residual=True),
        # the features of a test set by the served network, in the library's
        # own type
        dict(name="linear4_5000x784x2048_f32", kind="linear4", m=5000, k=784,
             n=2048, group=128, type="f32", act="gelu", residual=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: half of them multiples of 64, the rest as they
    come."""
    v = _log(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.5 and hi >= 64 else v


def draw(rng):
    kind = rng.choice(["grad_norm", "clipped_step", "group_norm",
                       "group_norm", "group_bwd", "group_bwd", "linear4",
                       "linear4", "linear4"])
    t = rng.choice(["f32", "bf16", "f16"])
    if kind in ("grad_norm", "clipped_step"):
        c = dict(kind=kind, d=_size(rng, 20, 1024), blocks=rng.randint(0, 12),
                 width=_size(rng, 32, 1536), classes=rng.randint(1, 20),
                 type=t, max_norm=rng.choice([0.1, 1.0, 100.0]),
                 grad_scale=rng.choice([1.0, 0.25, 2.0 ** -10]))
        if kind == "clipped_step":
            c["master"] = t != "f32" and rng.random() < 0.7
        return c
    if kind in ("group_norm", "group_bwd"):
        most = 5e7 if kind == "group_norm" else 2.5e7
        while True:
            n, s = _log(rng, 1, 4096), _log(rng, 1, 8192)
            groups, each = _log(rng, 1, 64), _log(rng, 1, 256)
            if rng.random() < 0.5:
                each = max(8, each // 8 * 8)
            if 8 <= groups * each <= 4096 and n * s * groups * each <= most:
                break
        c = dict(kind=kind, samples=n, positions=s, channels=groups * each,
                 groups=groups, type=t, act=rng.choice(ACTS))
        if kind == "group_bwd":
            c["residual"] = rng.random() < 0.5
        return c
    while True:
        m = _log(rng, 1, 8192) if rng.random() < 0.4 else _log(rng, 1, 64)
        k, n = _size(rng, 16, 16384), _size(rng, 16, 16384)
        if m * k * n <= 1.6e10 and k * n <= 6.7e7:
            break
    return dict(kind=kind, m=m, k=k, n=n, group=rng.choice([32, 64, 128]),
                type=t, act=rng.choice(ACTS), residual=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs


def _shapes(c):
    """The tensors of a feature network: first layer, blocks of norm and
    layer, head."""
    w = c["width"]
    block = [(w,), (w,), (w, w), (w,)]
    return ([(w, c["d"]), (w,)] + block * c["blocks"] +
            [(c["classes"], w), (c["classes"],)])


def _parts(c):
    """(first element, size) of each tensor in the flat states: every tensor
    begins at a multiple of BLOCK."""
    sizes = [math.prod(s) for s in _shapes(c)]
    at, out = 0, []
    for n in sizes:
        out.append((at, n))
        at += -(-n // BLOCK) * BLOCK
    return out, at


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[c["type"]]

    def normal(*shape, by=1.0, to=t):
        return torch.randn(shape, generator=g, device=DEV).mul_(by).to(to)

    def uniform(*shape, lo=0.0, hi=1.0, to=torch.float32):
        return (torch.rand(shape, generator=g, device=DEV) * (hi - lo)
                + lo).to(to)

    if c["kind"] in ("grad_norm", "clipped_step"):
        # gradients of a few 1e-3, times the loss scale
        by = 1e-3 / c["grad_scale"]
        s = dict(case=c, grads=[normal(*sh, by=by) for sh in _shapes(c)])
        if c["kind"] == "grad_norm":
            return s
        parts, total = _parts(c)
        s.update(params=[normal(*sh, by=0.05) for sh in _shapes(c)],
                 m=normal(total, by=5e-4, to=torch.float32),
                 v=normal(total, by=1e-3, to=torch.float32).square_(),
                 master=None)
        for a, n in parts:  # (what lies past a tensor's end stays 0)
            for x in (s["m"], s["v"]):
                x[a + n:a + -(-n // BLOCK) * BLOCK] = 0
        if c["master"]:
            s["master"] = torch.zeros(total, device=DEV)
            views = [s["master"][a:a + n].view(p.shape)
                     for (a, n), p in zip(parts, s["params"])]
            torch._foreach_copy_(views, s["params"])
        return s
    if c["kind"] in ("group_norm", "group_bwd"):
        shape = (c["samples"], c["positions"], c["channels"])
        # each sample and each channel has a level of its own
        x = normal(*shape, by=1.5, to=torch.float32)
        x += uniform(shape[0], 1, 1, lo=-1.0)
        x += uniform(shape[2], lo=-1.0)
        s = dict(case=c, X=x.to(t), w=(1 + normal(shape[2], by=0.1)).to(t),
                 b=normal(shape[2], by=0.1))
        if c["kind"] == "group_bwd":
            mean, rstd = _moments(_grouped(s["X"], c).double())
            s.update(mean=mean.float().view(shape[0], -1),
                     rstd=rstd.float().view(shape[0], -1), dY=normal(*shape),
                     res=normal(*shape) if c["residual"] else None)
        return s
    m, k, n = c["m"], c["k"], c["n"]
    W = normal(n, k, by=math.sqrt(1.0 / k))
    s = dict(case=c, X=normal(m, k), b=normal(n, by=0.1),
             R=normal(m, n) if c["residual"] else None)
    s["codes"], s["scales"] = _to4(W, c["group"])
    if own:
        from paper_1706_05544_amd import native as nv
        s["packed"] = nv.svm_pack_weights(W, c["group"])
    return s


# ------------------------------------------------- the definitions, by type


def _grouped(x, c):
    """samples x positions x groups x channels of a group"""
    return x.reshape(c["samples"], c["positions"], c["groups"], -1)


def _moments(x):
    mean = x.mean((1, 3), keepdim=True)
    var = (x - mean).square().mean((1, 3), keepdim=True)
    return mean, (var + EPS).rsqrt()


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return torch.tanh(z) if name == "tanh" else z


def _slope(name, z):
    if name == "gelu":
        return (0.5 * (1 + torch.erf(z * math.sqrt(0.5))) +
                z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)))
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return 1 - torch.tanh(z).square() if name == "tanh" else torch.ones_like(z)


def _to4(W, group):
    """The weights in 4 bits: (codes, two to a byte, a row's k rounded up to
    even; scales).  A group's scale is a sixth of its largest magnitude with
    six significant bits kept (in f16 in whole steps of 2^-23), so that a
    scale times a code is a value of the type; a code is a sign (bit 3) and
    the place in GRID that is nearest to the weight over the scale."""
    n, k = W.shape
    pad = torch.nn.functional.pad(W.float(), (0, -k % group))
    pad = pad.view(n, -1, group)
    top = pad.abs().amax(2)
    bits = (top / 6.0).view(torch.int32) & ~((1 << 18) - 1)
    s = bits.view(torch.float32)
    if W.dtype == torch.float16:
        s = torch.floor(s * 2.0 ** 23) * 2.0 ** -23
    x = torch.where(s[..., None] > 0, pad.abs() / s[..., None], 0)
    code = torch.zeros(x.shape, dtype=torch.uint8, device=W.device)
    for i, border in enumerate(BORDERS):
        code += x > border if i % 2 == 0 else x >= border
    code |= (pad < 0).to(torch.uint8) << 3
    code = code.view(n, -1)
    if code.shape[1] % 2:
        code = torch.nn.functional.pad(code, (0, 1))
    return code[:, 0::2] | (code[:, 1::2] << 4), s.to(W.dtype)


def _from4(codes, scales, k, group, dtype):
    """The weights that the codes stand for."""
    table = torch.tensor(GRID + tuple(-v for v in GRID), dtype=dtype,
                         device=codes.device)
    at = torch.stack([codes & 15, codes >> 4], 2).view(len(codes), -1)
    w = table[at.int()].view(len(codes), -1, group)
    return (w * scales.to(dtype)[..., None]).view(len(codes), -1)[:, :k]


# --------------------------------------------------------- the plain forms


def _plain_grad_norm(s):
    c = s["case"]
    # (a square is exact in 64 bits, and in reach)
    square = sum(g.double().square().sum() for g in s["grads"])
    norm = square.sqrt() * c["grad_scale"]
    factor = torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0)
    return norm.float(), factor.float()


def _flat(tensors, total):
    """The tensors one after another, each padded with zeros to a multiple of
    BLOCK, in 32 bits."""
    zeros = torch.zeros(BLOCK, device=DEV)
    pieces = [p for t in tensors for p in (
        t.reshape(-1).float(), zeros[:-t.numel() % BLOCK])]
    out = torch.cat(pieces)
    assert out.numel() == total
    return out


def _plain_clipped_step(s):
    c, h = s["case"], ADAM
    norm, factor = _plain_grad_norm(s)
    parts, total = _parts(c)
    g = _flat(s["grads"], total) * (c["grad_scale"] * factor)
    p = s["master"] if c["master"] else _flat(s["params"], total)
    s["m"].mul_(h["beta1"]).add_(g * (1 - h["beta1"]))
    s["v"].mul_(h["beta2"]).add_((g * g) * (1 - h["beta2"]))
    b1 = 1 - h["beta1"] ** h["step"]
    b2 = 1 - h["beta2"] ** h["step"]
    p = (p * (1 - h["lr"] * h["weight_decay"]) - (h["lr"] / b1) *
         (s["m"] / (torch.sqrt(s["v"]) * (1 / math.sqrt(b2)) + h["eps"])))
    if c["master"]:
        s["master"].copy_(p)
    torch._foreach_copy_(s["params"], [p[a:a + n].view(x.shape) for (a, n), x
                                       in zip(parts, s["params"])])
    return norm, factor, s["params"], s["m"], s["v"], s["master"]


def _plain_group_norm(s):
    c, x = s["case"], s["X"].float()
    xg = _grouped(x, c)
    mean, rstd = _moments(xg)
    z = ((xg - mean) * rstd).view(x.shape) * s["w"].float() + s["b"].float()
    n = c["samples"]
    return (_act(c["act"], z).to(s["X"].dtype), mean.view(n, -1),
            rstd.view(n, -1))


def _plain_group_bwd(s):
    c, t = s["case"], s["X"].dtype
    shape = s["X"].shape
    mean, rstd = (s[k].view(c["samples"], 1, -1, 1) for k in ("mean", "rstd"))
    w, b, dz = s["w"].float(), s["b"].float(), s["dY"].float()
    xh = ((_grouped(s["X"].float(), c) - mean) * rstd).view(shape)
    if c["act"] == "relu":
        # (which side of 0 the value lies on: in 64 bits)
        z = ((_grouped(s["X"].double(), c) - mean) * rstd.double()).view(
            shape) * w + b
        dz = torch.where(z > 0, dz, 0)
    else:
        dz = dz * _slope(c["act"], xh * w + b)
    a, xg = _grouped(dz * w, c), _grouped(xh, c)
    dx = rstd * (a - a.mean((1, 3), keepdim=True) -
                 xg * (a * xg).mean((1, 3), keepdim=True))
    dx = dx.view(shape)
    if s["res"] is not None:
        dx = dx + s["res"].float()
    return (dx.to(t), (dz * xh).sum((0, 1)).to(t), dz.sum((0, 1)).to(t))


def _plain_linear4(s):
    c, t = s["case"], TYPES[s["case"]["type"]]
    W = _from4(s["codes"], s["scales"], c["k"], c["group"], torch.float32)
    y = _act(c["act"], s["X"].float() @ W.t() + s["b"].float())
    if s["R"] is not None:
        y = y + s["R"].float()
    return y.to(t)


_PLAIN = dict(grad_norm=_plain_grad_norm, clipped_step=_plain_clipped_step,
              group_norm=_plain_group_norm, group_bwd=_plain_group_bwd,
              linear4=_plain_linear4)


# ---------------------------------------------------------- the library's


def _library(s):
    from paper_1706_05544_amd import native as nv

    c = s["case"]
    kind = c["kind"]
    if kind in ("grad_norm", "clipped_step"):
        norm, factor = nv.svm_grad_norm(s["grads"], c["max_norm"],
                                        grad_scale=c["grad_scale"])
        if kind == "grad_norm":
            return norm, factor
        nv.svm_adamw_step(s["params"], s["grads"], s["m"], s["v"],
                          master=s["master"], grad_scale=c["grad_scale"],
                          factor=factor, **ADAM)
        return norm, factor, s["params"], s["m"], s["v"], s["master"]
    if kind == "group_norm":
        return nv.svm_group_norm(s["X"], c["groups"], s["w"], s["b"],
                                 eps=EPS, act=c["act"], save=True)
    if kind == "group_bwd":
        return nv.svm_group_norm_backward(
            s["dY"], s["X"], c["groups"], s["mean"], s["rstd"], s["w"],
            s["b"], act=c["act"], residual=s["res"])
    return nv.svm_linear_packed(s["X"], s["packed"], s["b"], s["R"],
                                act=c["act"])


def run(state):
    if own:
        return _library(state)
    return _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------- work


def work(case):
    c = case
    e = {"f32": 4, "bf16": 2, "f16": 2}[c["type"]]
    kind = c["kind"]
    if kind in ("grad_norm", "clipped_step"):
        n = sum(size for _, size in _parts(c)[0])
        if kind == "grad_norm":
            return {"bytes": n * e + 8, "flops": 2 * n}
        # gradient read, weight written, what it comes from read (a master
        # copy is written too), two states read and written
        return {"bytes": n * (2 * e + (8 if c["master"] else e) + 16) + 8,
                "flops": 18 * n}
    if kind in ("group_norm", "group_bwd"):
        n = c["samples"] * c["positions"] * c["channels"]
        st = 8 * c["samples"] * c["groups"]
        if kind == "group_norm":
            return {"bytes": e * (2 * n + 2 * c["channels"]) + st,
                    "flops": 12 * n}
        return {"bytes": e * ((3 + c["residual"]) * n + 4 * c["channels"]) +
                st, "flops": 28 * n}
    m, k, n = c["m"], c["k"], c["n"]
    return {"bytes": n * ((k + 1) // 2) + e * (
        n * -(-k // c["group"]) + m * k + n + m * n * (1 + c["residual"])),
            "flops": 2 * m * n * k}


# --------------------------------------------------- definitions in 64 bits


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    d = lambda x: x.to(torch.float64)  # noqa: E731
    kind = c["kind"]
    if kind in ("grad_norm", "clipped_step"):
        # of one long vector, its largest magnitude taken out
        flat = torch.cat([d(g).flatten() for g in s["grads"]])
        top = flat.abs().max()
        norm = top * torch.linalg.vector_norm(flat / top) * c["grad_scale"]
        factor = (c["max_norm"] / norm).clamp(max=1.0)
        if kind == "grad_norm":
            return norm, factor
        return (norm, factor) + _exact_step(s, float(factor))
    if kind == "linear4":
        # decoded by the bits: two of exponent, one of significand
        q = torch.stack([s["codes"] % 16, s["codes"] // 16], -1).flatten(1)
        q = q[:, :c["k"]].long()
        e, f = (q >> 1) & 3, d(q & 1)
        w = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * 2.0 ** (d(e) - 1))
        w = torch.where(q >= 8, -w, w)
        by = d(s["scales"]).repeat_interleave(c["group"], 1)[:, :c["k"]]
        y = _act64(c["act"], d(s["X"]).matmul((w * by).t()) + d(s["b"]))[0]
        return y if s["R"] is None else y + d(s["R"])
    # samples x groups x (positions x channels of a group)
    n, p, ch, g = c["samples"], c["positions"], c["channels"], c["groups"]

    def rows(x):
        return d(x).view(n, p, g, ch // g).transpose(1, 2).reshape(n, g, -1)

    def back(x):
        return x.view(n, g, p, ch // g).transpose(1, 2).reshape(n, p, ch)

    x = rows(s["X"])
    size = x.shape[2]
    if kind == "group_norm":
        mean = x.sum(2) / size
        off = x - mean[..., None]
        rstd = 1 / torch.sqrt((off ** 2).sum(2) / size + EPS)
        z = back(off * rstd[..., None]) * d(s["w"]) + d(s["b"])
        return _act64(c["act"], z)[0], mean, rstd
    mean, rstd = d(s["mean"])[..., None], d(s["rstd"])[..., None]
    off = x - mean
    xh = back(off * rstd)
    dz = d(s["dY"]) * _act64(c["act"], xh * d(s["w"]) + d(s["b"]))[1]
    a = rows(dz * d(s["w"]))
    # dx = rstd (a_j - sum_k a_k (1 + xh_j xh_k) / size)
    sx = (a * off).sum(2, keepdim=True) * rstd ** 2 / size
    dx = back(rstd * (a - a.sum(2, keepdim=True) / size - off * sx))
    if c["residual"]:
        dx = dx + d(s["res"])
    return dx, (dz * xh).sum((0, 1)), dz.sum((0, 1))


def _act64(name, z):
    """(activation, its derivative)"""
    if name == "relu":
        return torch.relu(z), (z > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.erfc(z * -math.sqrt(0.5))
        return z * cdf, cdf + z * torch.exp(z * z / -2) / math.sqrt(
            2 * math.pi)
    if name == "silu":
        e = 1 / (1 + torch.exp(-z))
        return z * e, e + z * e * (1 - e)
    if name == "tanh":
        y = torch.tanh(z)
        return y, 1 - y * y
    return z, torch.ones_like(z)


def _exact_step(s, factor):
    c, h = s["case"], ADAM
    b1, b2 = h["beta1"], h["beta2"]
    new = [[], [], [], []]
    for i, (a, n) in enumerate(_parts(c)[0]):
        pad = -(-n // BLOCK) * BLOCK
        m, v = s["m"][a:a + pad].double(), s["v"][a:a + pad].double()
        g = torch.zeros(pad, dtype=torch.float64, device=m.device)
        g[:n] = s["grads"][i].double().flatten() * (c["grad_scale"] * factor)
        p = (s["master"][a:a + n] if c["master"]
             else s["params"][i].flatten()).double()
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g ** 2
        mh = m[:n] / (1 - b1 ** h["step"])
        vh = v[:n] / (1 - b2 ** h["step"])
        p = p - h["lr"] * (h["weight_decay"] * p + mh / (vh ** 0.5 + h["eps"]))
        full = torch.zeros(pad, dtype=torch.float64, device=m.device)
        full[:n] = p
        for to, x in zip(new, (p.view(s["params"][i].shape), m, v, full)):
            to.append(x)
    return (new[0], torch.cat(new[1]), torch.cat(new[2]),
            torch.cat(new[3]) if c["master"] else None)
