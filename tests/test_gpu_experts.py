"""Routing, linear layers over bins and their combination on the GPU against plain 64-bit
forms (experts_reference.py).

Tolerances count roundings.  u = eps / 2 of the 16-bit type is one rounding's relative
error, U = 2^-24 float32's.  A sum of m float32 products in any order is off by at most
(m + 2) U times the sum of the products' absolute values, S; activations and their
derivatives multiply an error of z by at most 1.13 and add at most 2^-19 (|z| + 1) of their
own (an approximation of erf within 1.5e-7, fast exponentials)."""
import ctypes
import math

import pytest
import torch

import experts_reference as R
from paper_2608_27888_amd import ntc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ntc.lib()
    return torch.device("cuda:0")


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """Half the spacing of the smallest numbers."""
    return torch.finfo(t).tiny * torch.finfo(t).eps / 2


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def strided(t, pad, dev, fill=math.nan):
    """The matrix on the device with `pad` more elements (NaN) behind every row."""
    if pad == 0:
        return t.to(dev)
    big = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=dev)
    big[:, :t.shape[1]] = t.to(dev)
    return big[:, :t.shape[1]]


def close(got, want, tol):
    got, want = got.cpu().double(), want.double()
    both = torch.isnan(got) & torch.isnan(want)
    equal = got == want  # infinities
    off = torch.where(both | equal, torch.zeros_like(want), (got - want).abs() - tol)
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0.0 and not torch.isnan(off).any(), worst


# ------------------------------------------------------------------------------ routing

ROUTES = [
    dict(n=1, E=1, k=1), dict(n=1, E=64, k=6), dict(n=7, E=8, k=8), dict(n=33, E=60, k=4),
    dict(n=130, E=65, k=3), dict(n=9, E=128, k=64), dict(n=50, E=40, k=40),
    dict(n=65, E=200, k=8), dict(n=5, E=1024, k=17), dict(n=6, E=257, k=2),
    dict(n=31, E=64, k=4, groups=(8, 3, 1)), dict(n=31, E=64, k=4, groups=(4, 2, 2), bias=True),
    dict(n=40, E=256, k=8, groups=(8, 4, 2), bias=True), dict(n=12, E=96, k=5, groups=(4, 1, 2)),
    dict(n=12, E=160, k=6, groups=(8, 3, 1), bias=True), dict(n=7, E=60, k=2, groups=(60, 5, 2)),
    dict(n=4, E=1024, k=8, groups=(16, 4, 2), bias=True), dict(n=21, E=48, k=5, bias=True),
    dict(n=9, E=12, k=3, groups=(2, 2, 2)), dict(n=70, E=32, k=4, groups=(8, 2, 2), bias=True),
    dict(n=19, E=512, k=6, groups=(2, 1, 2), bias=True), dict(n=3, E=640, k=6, groups=(5, 2, 1)),
]


def logits_for(c, seed, kind):
    g = gen(seed)
    l = torch.randn(c["n"], c["E"], generator=g) * 2
    if kind == "ties":  # few distinct values: many equal scores
        l = torch.randint(-2, 3, (c["n"], c["E"]), generator=g).float()
        l[l == 0] *= -1.0  # zeros of both signs
    if kind == "masked":  # rows with few, one or no experts left
        l[torch.rand(c["n"], c["E"], generator=g) < 0.7] = -math.inf
        l[0] = -math.inf
        if c["n"] > 3:
            l[1] = math.nan
            l[2, 1:] = math.nan
            l[3, : c["E"] // 2] = -3.0e38
    if kind == "extreme":
        l = torch.where(l > 1, torch.full_like(l, 60000.0), l)
        l = torch.where(l < -1, torch.full_like(l, -60000.0), l)
        l[0] = -60000.0
        if c["n"] > 2:
            l[1, 0], l[2] = math.inf, math.inf
    return l


@pytest.mark.parametrize("c", ROUTES, ids=str)
@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "extreme"])
def test_route(dev, c, kind):
    G, top, gt = c.get("groups", (1, 1, 1))
    for at, (score, renorm, dtype) in enumerate([("softmax", True, F32), ("sigmoid", True, BF16),
                                                 ("softmax", False, F16),
                                                 ("sigmoid", False, F32)]):
        l = logits_for(c, 11 + at, kind).to(dtype)
        bias = None
        if c.get("bias"):
            bias = 0.1 * torch.randn(c["E"], generator=gen(5))
            if kind == "masked":
                bias[c["E"] // 3] = -math.inf
                bias[c["E"] // 2] = math.nan
            if kind == "ties":
                bias = torch.zeros(c["E"])
        mask = torch.rand(c["n"], generator=gen(6)) > 0.2 if at % 2 else None
        opt = dict(score=score, n_groups=G, top_groups=top, group_top=gt, renormalize=renorm,
                   scale=2.5 if at else 1.0)
        ids, w = R.choose(l.double(), c["k"], bias=bias, mask=mask, **opt)
        got = ntc.route(strided(l, at, dev), c["k"], bias=None if bias is None else bias.to(dev),
                        mask=None if mask is None else mask.to(dev), **opt)
        assert torch.equal(got.ids.cpu(), ids)
        # exponentials of differences up to 70 (further apart underflows), sums of E terms
        close(got.weights, w, (70 + c["E"] + 16) * U * w + 1e-37)
        assert bool((got.weights.cpu()[ids < 0] == 0).all())


@pytest.mark.parametrize("E,k,groups", [(40, 5, (1, 1, 1)), (96, 6, (4, 2, 2)), (256, 8, (8, 4, 2)),
                                        (200, 16, (1, 1, 1)), (600, 7, (3, 2, 1))])
@pytest.mark.parametrize("biased", [True, False])
def test_route_close_values(dev, E, k, groups, biased):
    """Experts whose values agree in all but their last float32 bits, in twos and in threes:
    the order is float64's."""
    g = gen(E)
    n = 300
    l = torch.randn(n, E, generator=g)
    bias = 0.2 * torch.randn(E, generator=g) if biased else torch.zeros(E)
    for t in range(n):
        best = torch.sort(torch.sigmoid(l[t].double()) + bias.double(), descending=True).indices
        near = [best[int(torch.randint(0, k + 2, (1,), generator=g))]]
        near += [best[E // 2 + j] for j in range(1 + t % 2)]
        for e in near[1:]:
            if biased:
                s = torch.sigmoid(l[t, near[0]].double()) + bias[near[0]].double() - bias[e].double()
                if 0.01 < s < 0.99:
                    l[t, e] = torch.logit(s).float()
            else:
                l[t, e] = torch.nextafter(l[t, near[0]], torch.tensor([-9.0, 9.0][t // 2 % 2]))
    for score in ("sigmoid", "softmax"):
        opt = dict(score=score, n_groups=groups[0], top_groups=groups[1], group_top=groups[2])
        b = bias if biased else None
        ids, w = R.choose(l.double(), k, bias=b, **opt)
        got = ntc.route(l.to(dev), k, bias=None if b is None else b.to(dev), **opt)
        assert torch.equal(got.ids.cpu(), ids), score
        close(got.weights, w, (70 + E + 16) * U * w + 1e-37)


@pytest.mark.parametrize("c", ROUTES[:12], ids=str)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward(dev, c, score, renorm):
    for dtype, kind in ((F32, "plain"), (BF16, "ties"), (F16, "masked")):
        l = logits_for(c, 3, kind).to(dtype)
        ids = ntc.route(l.to(dev), c["k"], score=score).ids
        dw = torch.randn(c["n"], c["k"], generator=gen(9))
        dw[(ids < 0).cpu()] = math.nan  # empty slots take no part
        got = ntc.route_backward(strided(l, 3, dev), ids, dw.to(dev), score=score,
                                 renormalize=renorm, scale=1.5)
        assert got.dtype == dtype
        at = ids.cpu()
        live = (at >= 0).any(1)
        ld = l.double()
        ld = torch.where(live[:, None], ld, torch.zeros_like(ld)).requires_grad_(True)
        w = R.weights_of(ld, at, score, renorm, 1.5)
        g, = torch.autograd.grad((w * torch.where(at < 0, 0.0, dw.double())).sum(), ld)
        # a gradient is a sum of at most k + 1 terms of at most |scale p g|
        size = 1.5 * torch.where(at < 0, 0.0, dw.double().abs()).sum(1, keepdim=True)
        close(got, torch.nan_to_num(g), half(dtype) * g.abs().nan_to_num() + tiny(dtype)
              + (70 + c["E"] + 2 * c["k"] + 16) * U * size)


def test_route_backward_is_the_difference_quotient(dev):
    """Against differences of the forward pass itself, choice unchanged."""
    g = gen(2)
    l, dw = torch.randn(5, 24, generator=g), torch.randn(5, 4, generator=g)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            ids = ntc.route(l.to(dev), 4, score=score, renormalize=renorm).ids
            got = ntc.route_backward(l.to(dev), ids, dw.to(dev), score=score,
                                     renormalize=renorm).cpu()
            h = 2.0 ** -7
            for e in range(24):
                w = []
                for sign in (1, -1):
                    moved = l.clone()
                    moved[:, e] += sign * h
                    w.append(R.weights_of(moved.double(), ids.cpu(), score, renorm, 1.0))
                diff = ((w[0] - w[1]) / (2 * h) * dw.double()).sum(1)
                # third derivatives of softmax and sigmoid weights are at most 1: h^2 / 6 each
                assert bool(((got[:, e] - diff).abs() <= h * h / 6 * dw.abs().sum(1)
                             + 1e-5).all())


def test_route_backward_same_expert_twice(dev):
    l = torch.tensor([[0.5, -1.0, 2.0, 0.0]])
    ids = torch.tensor([[2, 2, 7]], dtype=torch.int32)  # 7: out of range, skipped
    dw = torch.tensor([[1.0, 0.5, math.nan]])
    s = torch.sigmoid(l.double())[0, 2]
    got = ntc.route_backward(l.to(dev), ids.to(dev), dw.to(dev), score="sigmoid",
                             renormalize=False).cpu()
    close(got[0, 2], 1.5 * s * (1 - s), torch.tensor(8 * U))
    assert got[0, [0, 1, 3]].tolist() == [0.0, 0.0, 0.0]


# ------------------------------------------------------------------------- linear layers

LINEAR = [
    dict(n=1, i=64, o=64), dict(n=1, i=1, o=1), dict(n=3, i=7, o=5), dict(n=16, i=512, o=96),
    dict(n=17, i=1000, o=130), dict(n=65, i=72, o=257), dict(n=128, i=128, o=128),
    dict(n=129, i=136, o=140), dict(n=300, i=264, o=520, pad=8), dict(n=130, i=65, o=64, pad=3),
    dict(n=64, i=2048, o=33), dict(n=520, i=320, o=300, pad=4), dict(n=5, i=4104, o=264),
    dict(n=700, i=640, o=512), dict(n=257, i=96, o=1030),
    # experts
    dict(n=1, k=2, E=4, i=64, o=32), dict(n=9, k=3, E=5, i=40, o=24, div=3),
    dict(n=200, k=2, E=3, i=128, o=136, div=2), dict(n=90, k=4, E=16, i=72, o=70, div=4, pad=1),
    dict(n=500, k=1, E=2, i=256, o=264), dict(n=37, k=8, E=64, i=512, o=128, div=8),
    dict(n=300, k=5, E=300, i=64, o=64, div=5), dict(n=333, k=3, E=7, i=200, o=56, div=3, align=1),
    dict(n=64, k=2, E=4, i=64, o=64, align=1024), dict(n=900, k=2, E=4, i=320, o=264, div=2),
]


def linear_case(c, dtype, seed, dev):
    """Host tensors of a case: x, weight [E][out][in], bias, expert of every slot, div, bins."""
    g = gen(seed)
    E, k, div = c.get("E", 1), c.get("k", 1), c.get("div", 1)
    n = c["n"] * k
    x = torch.randn(n // div, c["i"], generator=g).to(dtype)
    w = (torch.randn(E, c["o"], c["i"], generator=g) * c["i"] ** -0.5).to(dtype)
    b = torch.randn(E, c["o"], generator=g).to(dtype)
    expert, bins = torch.zeros(n, dtype=torch.int64), None
    if "E" in c:
        # popular experts, experts without slots, slots in no bin
        expert = torch.randint(0, E + 1, (n,), generator=g)
        expert[torch.rand(n, generator=g) < 0.3] = E // 2
        ids = torch.where(expert >= E, -1, expert).to(torch.int32)
        expert = torch.where(expert >= E, -1, expert)
        bins = ntc.build_bins(ids.to(dev), torch.arange(E, dtype=torch.int32, device=dev), E,
                              align=c.get("align", 64))
    return x, w, b, expert, div, bins


@pytest.mark.parametrize("c", LINEAR, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_linear(dev, c, dtype):
    x, w, b, expert, div, bins = linear_case(c, dtype, 21, dev)
    n, o, pad = expert.numel(), c["o"], c.get("pad", 0)
    wd = w.to(dev) if bins is not None else w[0].to(dev)
    xs = strided(x, pad, dev)
    inside = expert >= 0
    for at, act in enumerate(("none", "relu", "leaky_relu", "gelu", "silu")):
        slope = 0.1 if act == "leaky_relu" else None
        bias = b if at % 2 else None
        to = F32 if at in (1, 3) else dtype
        res = torch.randn(n, o, generator=gen(4)).to(to) if at >= 2 else None
        pre = strided(torch.full((n, o), 7.0, dtype=dtype), pad, dev) if at in (0, 3, 4) else None
        out = strided(torch.full((n, o), 7.0, dtype=to), pad, dev, 5.0)
        got = ntc.linear(xs, wd, None if bias is None else (b if bins is not None else b[0]).to(dev),
                         residual=None if res is None else strided(res, pad, dev),
                         activation=act, leaky_slope=slope, bins=bins, slots_per_row=div, out=out,
                         pre=pre)
        assert got is out
        y, z, size = R.linear(x.double(), w.double(), None if bias is None else b.double(),
                              expert, div, act, slope or 0.0)
        if res is not None:
            y = y + res.double()
        zoff = (c["i"] + 4) * U * size
        tol = 1.13 * zoff + 2.0 ** -19 * (z.abs() + 1) + 4 * U * y.abs()
        if to != F32:
            tol = tol + half(to) * (y.abs() + tol) + tiny(to)
        close(got[inside.to(dev)], y[inside], tol[inside])
        assert bool((got[~inside.to(dev)] == 7.0).all())
        if pre is not None:
            close(pre[inside.to(dev)], z[inside],
                  (zoff + half(dtype) * (z.abs() + zoff) + tiny(dtype))[inside])
            assert bool((pre[~inside.to(dev)] == 7.0).all())
        if pad:  # what lies between the rows
            assert bool((out.as_strided((n - 1, pad), (o + pad, 1), o) == 5.0).all())


@pytest.mark.parametrize("c", LINEAR, ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_linear_backward(dev, c, dtype):
    x, w, _, expert, div, bins = linear_case(c, dtype, 22, dev)
    n, o, i, pad = expert.numel(), c["o"], c["i"], c.get("pad", 0)
    wd = w.to(dev) if bins is not None else w[0].to(dev)
    for at, act in enumerate(("none", "relu", "gelu", "silu", "leaky_relu")):
        slope = 0.1 if act == "leaky_relu" else None
        from_f32, grad = (F32 if at in (1, 3) else dtype), (F32 if at in (0, 1, 4) else dtype)
        dy = torch.randn(n, o, generator=gen(8)).to(from_f32)
        pre = torch.randn(n, o, generator=gen(9)).to(dtype)
        pre[::3, ::2] = 0.0
        g = ntc.linear_backward(strided(dy, pad, dev), strided(x, pad, dev), wd,
                                pre=None if act == "none" else strided(pre, pad, dev),
                                activation=act, leaky_slope=slope, bins=bins, slots_per_row=div,
                                grad_dtype=grad)
        dz = dy.double()
        if act != "none":
            dz = dz * R.act_slope(pre.double(), act, slope or 0.0)
        # dz is rounded to the layer's type, after the derivative's own error
        dzoff = half(dtype) * 1.0001 * dz.abs() + 2.0 ** -18 * dy.double().abs() + tiny(dtype)
        if act in ("none", "relu") and from_f32 == dtype:
            dzoff = torch.zeros_like(dz)
        want, size = R.linear_grads(dz, x.double(), w.double(), expert, div)
        _, off = R.linear_grads(dzoff, x.double(), w.double(), expert, div)
        slots = torch.bincount(expert[expert >= 0], minlength=w.shape[0]).double()
        terms = [o, slots[:, None, None], slots[:, None]]
        for j, (name, t) in enumerate((("x", dtype), ("weight", grad), ("bias", grad))):
            got = getattr(g, name)
            assert got.dtype == t
            want_j = want[j] if name == "x" or bins is not None else want[j][0]
            tol = off[j] + (terms[j] + 4 + div) * U * (size[j] + off[j])
            tol = tol if name == "x" or bins is not None else tol[0]
            if t != F32:
                tol = tol + half(t) * (want_j.abs() + tol) + tiny(t)
            close(got, want_j, tol)


def test_linear_gradients_one_by_one(dev):
    """Any subset of the gradients, and none of a call without rows."""
    g = gen(1)
    x, w = torch.randn(70, 64, generator=g).to(BF16).to(dev), torch.randn(96, 64, generator=g).to(BF16).to(dev)
    dy = torch.randn(70, 96, generator=g).to(BF16).to(dev)
    full = ntc.linear_backward(dy, x, w)
    for keep in ("x", "weight", "bias"):
        part = ntc.linear_backward(dy, x, w, input_grad=keep == "x", weight_grad=keep == "weight",
                                   bias_grad=keep == "bias")
        for name in ("x", "weight", "bias"):
            if name == keep:
                assert torch.equal(getattr(part, name), getattr(full, name))
            else:
                assert getattr(part, name) is None
    empty = ntc.linear_backward(dy[:0], x[:0], w)
    assert empty.x.shape == (0, 64) and not bool(empty.weight.any()) and not bool(empty.bias.any())
    assert ntc.linear(x[:0], w).shape == (0, 96)


def test_linear_backward_is_the_difference_quotient(dev):
    """<gradient, direction> against differences of the 64-bit forward pass, through GELU."""
    g = gen(14)
    x, w = torch.randn(6, 24, generator=g).to(F16), (torch.randn(1, 16, 24, generator=g) / 5).to(F16)
    b, dy = torch.randn(1, 16, generator=g).to(F16), torch.randn(6, 16, generator=g).to(F16)
    expert = torch.zeros(6, dtype=torch.int64)
    pre = torch.empty(6, 16, dtype=F16, device=dev)
    ntc.linear(x.to(dev), w[0].to(dev), b[0].to(dev), activation="gelu", pre=pre)
    got = ntc.linear_backward(dy.to(dev), x.to(dev), w[0].to(dev), pre=pre, activation="gelu")
    h = 1e-4
    for name, t in (("x", x), ("weight", w), ("bias", b)):
        d = torch.randn(t.shape, generator=g).double()
        loss = []
        for sign in (h, -h):
            a = {"x": x.double(), "weight": w.double(), "bias": b.double()}
            a[name] = a[name] + sign * d
            y = R.linear(a["x"], a["weight"], a["bias"], expert, 1, "gelu")[0]
            loss.append((y * dy.double()).sum())
        diff = (loss[0] - loss[1]) / (2 * h)
        mine = (getattr(got, name).cpu().double().view(t.shape) * d).sum()
        # three roundings (pre, dz, the gradient) of each of the summed terms; the rounding
        # of pre moves a derivative by at most 0.8 |pre| u
        size = {"x": lambda: dy.double().abs() @ w[0].double().abs() * d.abs(),
                "weight": lambda: dy.double().abs().t() @ x.double().abs() * d.abs()[0],
                "bias": lambda: dy.double().abs().sum(0) * d.abs()[0]}[name]().sum()
        top = 1.13 * 2 + 0.8 * pre.abs().max().item()
        assert abs(mine - diff) <= top * half(F16) * size + 1e-6


def test_linear_keeps_infinities_apart(dev):
    """An infinity or NaN in one row reaches that row only; rows behind the last slot and
    columns behind the last value are never multiplied in."""
    g = gen(3)
    x, w = torch.randn(40, 72, generator=g).to(BF16), torch.randn(50, 72, generator=g).to(BF16)
    ref = ntc.linear(x.to(dev), w.to(dev))
    bad = x.clone()
    bad[7], bad[20, 3] = math.nan, math.inf
    got = ntc.linear(strided(bad, 8, dev), w.to(dev))
    rest = [r for r in range(40) if r not in (7, 20)]
    assert torch.equal(got[rest], ref[rest])
    assert bool(torch.isnan(got[7]).all()) and not bool(torch.isfinite(got[20]).any())
    dy = torch.randn(40, 50, generator=g).to(BF16)
    dy[7], dy[20] = 0, 0
    ids = torch.zeros(40, dtype=torch.int32)
    ids[7] = ids[20] = -1  # the same rows in no bin
    bins = ntc.build_bins(ids.to(dev), torch.zeros(1, dtype=torch.int32, device=dev), 1)
    d = ntc.linear_backward(dy.to(dev), strided(bad, 8, dev), w[None].to(dev), bins=bins)
    e = ntc.linear_backward(dy.to(dev), x.to(dev), w[None].to(dev), bins=bins)
    for a, c in ((d.x, e.x), (d.weight, e.weight), (d.bias, e.bias)):
        assert torch.equal(a, c) and bool(torch.isfinite(a).all())
    assert not bool(d.x[7].any()) and not bool(d.x[20].any())


def test_activations_of_infinities(dev):
    """Limits instead of infinity times zero, and NaN stays NaN; one row and a whole tile."""
    b = torch.tensor([math.inf, -math.inf, math.nan, 20000.0, -20000.0, 0.0, 3.0, -3.0])
    g = torch.tensor([1.0, 0.0, math.nan, 1.0, 0.0])
    for dtype in (F16, BF16):
        bd = b.to(dtype).to(dev)
        for n in (1, 200):
            x, w = torch.zeros(n, 64, dtype=dtype, device=dev), torch.zeros(8, 64, dtype=dtype, device=dev)
            dy = torch.ones(n, 8, dtype=dtype, device=dev)
            pre = bd.expand(n, 8).contiguous()
            for act in ("relu", "gelu", "silu"):
                y = ntc.linear(x, w, bd, activation=act).cpu().float()
                assert bool((y[:, 0] == math.inf).all()) and not bool(y[:, 1].any())
                assert bool(torch.isnan(y[:, 2]).all())
                assert bool((y[:, 3] == bd[3].float().item()).all()) and not bool(y[:, 4:6].any())
                d = ntc.linear_backward(dy, x, w, pre=pre, activation=act, input_grad=False,
                                        weight_grad=False, grad_dtype=F32).bias.cpu()
                want = n * g
                if act == "relu":  # NaN is not above 0
                    want[2] = 0.0
                assert torch.equal(torch.nan_to_num(d[:5], nan=-1.0), torch.nan_to_num(want, nan=-1.0))


# --------------------------------------------------------------------------- combination


@pytest.mark.parametrize("n,k,dim,pad", [(1, 1, 1, 0), (1, 8, 64, 0), (5, 3, 65, 0), (33, 2, 256, 8),
                                         (7, 8, 1000, 0), (130, 4, 2056, 0), (9, 64, 24, 1),
                                         (300, 6, 520, 3), (17, 5, 4096, 4)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_combine(dev, n, k, dim, pad, dtype):
    g = gen(n + k)
    rows, res = torch.randn(n * k, dim, generator=g).to(dtype), torch.randn(n, dim, generator=g).to(dtype)
    w, dout = torch.randn(n, k, generator=g), torch.randn(n, dim, generator=g).to(dtype)
    ids = torch.randint(0, 9, (n, k), generator=g).to(torch.int32)
    ids[torch.rand(n, k, generator=g) < 0.3] = -1  # ids of 8 are out of range of 8 experts
    gone = (ids < 0) | (ids >= 8)
    rows[gone.view(-1)] = math.nan  # skipped slots are not looked at
    w[gone] = math.nan
    for weights, at, residual in ((w, ids, res), (w, ids, None), (None, ids, res), (w, None, None)):
        r = rows.double().view(n, k, dim)
        live = torch.ones(n, k, dtype=torch.bool) if at is None else ~gone
        ww = torch.ones(n, k).double() if weights is None else weights.double()
        if at is None:  # everything takes part: no NaN
            r, ww = torch.nan_to_num(r), torch.nan_to_num(ww)
        terms = torch.where(live[..., None], r * ww[..., None], 0.0)
        want = terms.sum(1) + (0 if residual is None else residual.double())
        size = terms.abs().sum(1) + (0 if residual is None else residual.double().abs())
        dd = dict(weights=None if weights is None else (weights if at is not None else torch.nan_to_num(weights)).to(dev),
                  ids=None if at is None else at.to(dev), n_experts=8, k=k)
        src = strided(rows if at is not None else torch.nan_to_num(rows), pad, dev)
        got = ntc.combine(src, residual=None if residual is None else strided(residual, pad, dev), **dd)
        rounding = half(dtype) if dtype != F32 else 0.0
        close(got, want, (k + 2) * U * size + rounding * want.abs() * 1.001 + tiny(dtype))
        drows, dw = ntc.combine_backward(strided(dout, pad, dev), src, **dd)
        dr = torch.where(live[..., None], ww[..., None] * dout.double()[:, None], 0.0).view(n * k, dim)
        close(drows, dr, (U + rounding) * 1.001 * dr.abs() + tiny(dtype))
        prod = torch.where(live[..., None], r * dout.double()[:, None], 0.0)
        close(dw, prod.sum(2), (dim + 2) * U * prod.abs().sum(2))
        only, none = ntc.combine_backward(strided(dout, pad, dev), src, weights_grad=False, **dd)
        assert none is None and torch.equal(only, drows)
        none, only = ntc.combine_backward(strided(dout, pad, dev), src, rows_grad=False, **dd)
        assert none is None and torch.equal(only, dw)


def test_combine_in_place(dev):
    g = gen(8)
    rows, res = torch.randn(64, 128, generator=g).to(BF16).to(dev), torch.randn(16, 128, generator=g).to(BF16).to(dev)
    w = torch.rand(16, 4, generator=g).to(dev)
    want = ntc.combine(rows, w, residual=res)
    assert ntc.combine(rows, w, residual=res, out=res) is res
    assert torch.equal(want, res)


# ------------------------------------------------------------------------------ together


class Mixture:
    """A routed layer of two products an expert, forward and backward, by the library's calls."""

    def __init__(self, dev, n, d, f, E, k, dtype, seed=31):
        g = gen(seed)
        self.k, self.E = k, E
        self.x = torch.randn(n, d, generator=g).to(dtype).to(dev)
        self.logits = torch.randn(n, E, generator=g).to(dev)
        self.w1 = (torch.randn(E, f, d, generator=g) * d ** -0.5).to(dtype).to(dev)
        self.b1 = torch.randn(E, f, generator=g).to(dtype).to(dev)
        self.w2 = (torch.randn(E, d, f, generator=g) * f ** -0.5).to(dtype).to(dev)
        self.b2 = torch.randn(E, d, generator=g).to(dtype).to(dev)
        self.dout = torch.randn(n, d, generator=g).to(dtype).to(dev)
        self.mask = (torch.rand(n, generator=g) > 0.1).to(dev)
        self.identity = torch.arange(E, dtype=torch.int32, device=dev)

    def run(self):
        n, (E, f, d) = self.x.shape[0], self.w1.shape
        r = ntc.route(self.logits, self.k, mask=self.mask)
        bins = ntc.build_bins(r.ids, self.identity, E)
        pre = torch.empty(n * self.k, f, dtype=self.x.dtype, device=self.x.device)
        h = ntc.linear(self.x, self.w1, self.b1, activation="silu", bins=bins,
                       slots_per_row=self.k, pre=pre)
        y = ntc.linear(h, self.w2, self.b2, bins=bins)
        out = ntc.combine(y, r.weights, ids=r.ids, n_experts=E, residual=self.x)
        dy, dweights = ntc.combine_backward(self.dout, y, r.weights, ids=r.ids, n_experts=E)
        g2 = ntc.linear_backward(dy, h, self.w2, bins=bins)
        g1 = ntc.linear_backward(g2.x, self.x, self.w1, pre=pre, activation="silu", bins=bins,
                                 slots_per_row=self.k)
        dlogits = ntc.route_backward(self.logits, r.ids, dweights)
        return [out, r.ids, r.weights, g1.x + self.dout, dlogits, g1.weight, g1.bias, g2.weight,
                g2.bias]

    def reference(self, ids):
        """The same by automatic differentiation in 64 bits, the choice given."""
        at = ids.cpu()
        v = [t.cpu().double().requires_grad_(True) for t in
             (self.x, self.logits, self.w1, self.b1, self.w2, self.b2)]
        x, l, w1, b1, w2, b2 = v
        picked = torch.where(at >= 0, l.gather(1, at.clamp(min=0).long()), -1e30)
        w = torch.where(at >= 0, torch.softmax(picked, 1), 0.0)
        out = x
        for e in range(self.E):
            t, j = torch.nonzero(at == e, as_tuple=True)
            if t.numel():
                z = x[t] @ w1[e].t() + b1[e]
                y = (z * torch.sigmoid(z)) @ w2[e].t() + b2[e]
                out = out.index_add(0, t, y * w[t, j][:, None])
        grads = torch.autograd.grad((out * self.dout.cpu().double()).sum(), v)
        return [out.detach(), at, w.detach(), grads[0], grads[1], grads[2], grads[3], grads[4],
                grads[5]]


@pytest.mark.parametrize("n,d,f,E,k", [(1, 64, 32, 8, 2), (70, 128, 136, 8, 2), (257, 200, 72, 20, 4)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_mixture_together(dev, n, d, f, E, k, dtype):
    """Routing, binning, both products, combination and every gradient, as a training step
    uses them.  Every 16-bit value on the way is off by u; a gradient passes at most six of
    them (h, y, dy, dz, the slot's part, the result), so errors are at most 16 u of the root
    mean square that a tensor's own values have (independent roundings add up far less)."""
    m = Mixture(dev, n, d, f, E, k, dtype)
    got = m.run()
    want = m.reference(got[1])
    assert torch.equal(got[1].cpu() < 0, ~m.mask.cpu()[:, None].expand(n, k))
    for i, (a, b) in enumerate(zip(got, want)):
        if i == 1:
            continue
        a, b = a.cpu().double(), b.double()
        assert bool(torch.isfinite(a).all()), i
        scale = b.pow(2).mean().sqrt().item()
        assert (a - b).pow(2).mean().sqrt().item() <= 16 * half(dtype) * scale + 1e-12, i


def test_same_bits_again_and_on_streams(dev):
    """Runs give equal bits: again, on two side streams at once, and in a captured graph
    replayed between eager runs."""
    ms = [Mixture(dev, 150, 128, 96, 12, 3, BF16, 41), Mixture(dev, 90, 64, 200, 5, 2, F16, 42)]
    ref = [m.run() for m in ms]
    torch.cuda.synchronize()

    def same(a, b):
        return all(torch.equal(p, q) for p, q in zip(a, b))

    side = [torch.cuda.Stream(dev), torch.cuda.Stream(dev)]
    for _ in range(3):
        got = []
        for s, m in zip(side, ms):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(m.run())
        torch.cuda.synchronize()
        assert same(got[0], ref[0]) and same(got[1], ref[1])
    graphs = []
    for s, m in zip(side, ms):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = m.run()
        graphs.append((graph, outs))
    for rep in range(3):
        for graph, outs in graphs:
            for t in outs:
                t.zero_()
            graph.replay()
        assert same(ms[0].run(), ref[0])
        torch.cuda.synchronize()
        assert same(graphs[0][1], ref[0]) and same(graphs[1][1], ref[1])


def test_stream_argument(dev):
    """A call on a stream of its own, its inputs dropped right after."""
    g = gen(6)
    x, w = torch.randn(512, 512, generator=g).to(BF16), torch.randn(512, 512, generator=g).to(BF16)
    ref = ntc.linear(x.to(dev), w.to(dev), activation="gelu")
    side = torch.cuda.Stream(dev)
    for _ in range(4):
        a, b = x.to(dev), w.to(dev)
        side.wait_stream(torch.cuda.current_stream())
        got = ntc.linear(a, b, activation="gelu", stream=side)
        del a, b
        torch.zeros(512, 512, dtype=BF16, device=dev).fill_(9.0)  # would take freed memory
        side.synchronize()
        assert torch.equal(got, ref)


def test_rows_past_four_gib(dev):
    """Rows more than 2^32 bytes behind the first: offsets are 64-bit."""
    n, d, k = 300_000, 4096, 2  # 300,000 items of 8 KB, twice that for the slots
    rows = torch.zeros(n * k, d, dtype=BF16, device=dev)
    rows[-1], rows[-2] = 1.0, 2.0
    out = ntc.combine(rows, k=k)
    assert bool((out[-1] == 3.0).all()) and not bool(out[:-1].any())
    w = torch.zeros(8, d, dtype=BF16, device=dev)
    w[3, 5] = 1.0
    rows[-1, 5] = 4.0
    y = ntc.linear(rows, w)
    assert y[-1].tolist() == [0, 0, 0, 4.0, 0, 0, 0, 0] and y[-2, 3] == 2.0
    assert not bool(y[:-2].any())


def test_gathered_rows_past_four_gib(dev):
    """Rows by slot from a matrix of more than 4 GiB, forward and both gradients."""
    n, d, o = 600_000, 4096, 16
    g = gen(12)
    x = torch.zeros(n, d, dtype=BF16, device=dev)
    ids = torch.full((n,), -1, dtype=torch.int32)
    picks = torch.tensor([0, 1, 17, n // 2, n - 130, n - 2, n - 1])
    ids[picks] = torch.tensor([0, 1, 1, 0, 1, 1, 0], dtype=torch.int32)
    rows = torch.randn(len(picks), d, generator=g).to(BF16)
    x[picks.to(dev)] = rows.to(dev)
    w = torch.randn(2, o, d, generator=g).to(BF16)
    dy = torch.zeros(n, o, dtype=BF16, device=dev)
    dys = torch.randn(len(picks), o, generator=g).to(BF16)
    dy[picks.to(dev)] = dys.to(dev)
    identity = torch.arange(2, dtype=torch.int32, device=dev)
    bins = ntc.build_bins(ids.to(dev), identity, 2)
    y = ntc.linear(x, w.to(dev), bins=bins)
    grads = ntc.linear_backward(dy, x, w.to(dev), bins=bins)
    # the same slots alone
    small = ntc.build_bins(ids[picks].to(dev), identity, 2)
    assert torch.equal(y[picks.to(dev)], ntc.linear(rows.to(dev), w.to(dev), bins=small))
    alone = ntc.linear_backward(dys.to(dev), rows.to(dev), w.to(dev), bins=small)
    assert torch.equal(grads.x[picks.to(dev)], alone.x)
    assert int(grads.x.any(1).sum()) == len(picks)
    assert torch.equal(grads.weight, alone.weight) and torch.equal(grads.bias, alone.bias)
    # one layer over all rows: the other rows' gradients are 0
    dense = ntc.linear_backward(dy, x, w[0].to(dev))
    alone = ntc.linear_backward(dys.to(dev), rows.to(dev), w[0].to(dev))
    assert torch.equal(dense.x[picks.to(dev)], alone.x)
    assert int(dense.x.any(1).sum()) == len(picks)
    # the same products and zeros, in float32 in another order
    size = dys.double().abs().t() @ rows.double().abs()
    close(dense.weight, alone.weight.cpu(), 2 * half(BF16) * alone.weight.cpu().double().abs()
          + 2 * (len(picks) + 2) * U * size)


def test_outputs_on_another_stream(dev):
    """What a call on another stream returns isn't memory that earlier work of the current
    stream still writes to."""
    g = gen(12)
    l = torch.randn(4096, 64, generator=g).to(dev)
    x, w = (torch.randn(512, 512, generator=g).to(BF16).to(dev) for _ in range(2))
    rows = torch.randn(4096 * 2, 8, generator=g).to(dev)
    side = torch.cuda.Stream(dev)
    long = torch.randn(8192, 8192, device=dev).to(BF16)
    calls = [lambda s: ntc.route(l, 8, stream=s).ids, lambda s: ntc.linear(x, w, stream=s),
             lambda s: ntc.linear_backward(x, x, w, stream=s).weight,
             lambda s: ntc.combine(rows, k=2, stream=s)]
    for call in calls:
        want = call(None)
        old = torch.empty_like(want)
        torch.cuda.synchronize()
        for _ in range(8):
            long @ long
        old.fill_(9)  # behind the products
        del old
        got = call(side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def layer_args(x, w, n, div, dy, dx=None, dw=None, db=None):
    """A backward call's arguments without the binding: one layer, no activation."""
    t = ntc.TYPES[x.dtype]
    p = lambda v: None if v is None else v.data_ptr()
    layer = ntc.LinearLayer(1, w.shape[1], w.shape[0], t, w.data_ptr(), None)
    rows = ntc.LinearRows(n, p(x), w.shape[1], div, None, None, 0)
    grads = ntc.LinearGradsArgs(p(dy), w.shape[0], t, p(dx), w.shape[1], p(dw), p(db), t)
    return ctypes.byref(layer), ctypes.byref(rows), None, ctypes.byref(grads)


def test_no_rows_with_a_workspace(dev):
    """Without rows none is needed, but one may be given."""
    x, w, dy = (torch.ones(s, dtype=BF16, device=dev) for s in ((1, 64), (96, 64), (1, 96)))
    dw, db = torch.ones(96, 64, dtype=BF16, device=dev), torch.ones(96, dtype=BF16, device=dev)
    space = torch.empty(256, dtype=torch.uint8, device=dev)
    args = layer_args(x, w, 0, 1, dy, None, dw, db)
    assert ntc.lib().ntc_linear_backward_workspace_bytes(*args) == 0
    assert ntc.lib().ntc_linear_backward(*args, space.data_ptr(), 256,
                                         torch.cuda.current_stream().cuda_stream) == 0
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("div", [6, 1 << 20, 2 ** 31 - 1])
def test_more_slots_a_row_than_there_are(dev, div):
    """The last row's slots end with the call's; the rest costs neither time nor memory."""
    g = gen(13)
    n = 5
    x = torch.randn(1, 64, generator=g).to(BF16).to(dev)
    w = torch.randn(96, 64, generator=g).to(BF16).to(dev)
    dy = torch.randn(n, 96, generator=g).to(BF16).to(dev)
    want = ntc.linear_backward(dy, x, w, slots_per_row=n)
    got = [torch.full_like(t, 9.0) for t in (want.x, want.weight, want.bias)]
    args = layer_args(x, w, n, div, dy, *got)
    size = ntc.lib().ntc_linear_backward_workspace_bytes(*args)
    assert size < 1 << 16
    space = torch.empty(size, dtype=torch.uint8, device=dev)
    assert ntc.lib().ntc_linear_backward(*args, space.data_ptr(), size,
                                         torch.cuda.current_stream().cuda_stream) == 0
    for a, b in zip(got, (want.x, want.weight, want.bias)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("wide", ["dy", "x"])
def test_steps_past_the_end_of_four_gib(dev, wide):
    """9 steps of 64 rows whose end is the first byte past 4 GiB: what steps past it would
    read where offsets start over is NaN."""
    g = gen(14)
    n, stride = 576, 3728272
    assert n * stride * 2 - 2 ** 32 == 2048
    dy, x = (torch.randn(n, 64, generator=g).to(BF16).to(dev) for _ in range(2))
    w = torch.randn(64, 64, generator=g).to(BF16).to(dev)
    want = ntc.linear_backward(dy, x, w, grad_dtype=F32)
    far = torch.full((n, stride), math.nan, dtype=BF16, device=dev)
    far[:, :64] = dy if wide == "dy" else x
    rows = far[:, :64]
    got = ntc.linear_backward(rows if wide == "dy" else dy, rows if wide == "x" else x, w,
                              grad_dtype=F32)
    # sums of 576 products in another order
    S = dy.double().abs().T @ x.double().abs()
    assert bool(((got.weight - want.weight).abs() <= 2 * 578 * U * S).all())
    assert torch.equal(got.x, want.x)


@pytest.mark.parametrize("counts", [[8400], [9700], [12000], [5000, 301, 3100], [9000, 301, 3100], [4096, 4096],
                                    [8192 + 4096 + 1, 0, 5]], ids=str)
@pytest.mark.parametrize("o,i", [(2040, 1032), (1032, 2040)])
def test_last_round_of_tiles(dev, counts, o, i):
    """More 256 x 256 tiles than one round of the GPU: the rest of them few, many, none."""
    g = torch.Generator(dev)
    g.manual_seed(15)
    E, n, extra = len(counts), sum(counts), 7 if len(counts) > 1 else 0
    expert = torch.repeat_interleave(torch.arange(E, device=dev), torch.tensor(counts, device=dev))
    expert = torch.cat([expert, torch.full((extra,), -1, device=dev)])
    expert = expert[torch.randperm(n + extra, generator=g, device=dev)].contiguous()
    n += extra
    x, dy = (torch.randn(n, d, generator=g, device=dev).to(BF16) for d in (i, o))
    w = torch.randn(E, o, i, generator=g, device=dev).to(BF16)
    bins = None
    if E > 1:
        bins = ntc.build_bins(expert.to(torch.int32), torch.arange(E, dtype=torch.int32, device=dev), E)
    w1 = w[0] if bins is None else w
    y = torch.full((n, o), 7.0, device=dev)
    ntc.linear(x, w1, bins=bins, out=y)
    dx = ntc.linear_backward(dy, x, w1, bins=bins, weight_grad=False, bias_grad=False).x
    for e in range(E):
        s = expert == e
        for got, rows, m, terms in ((y[s], x[s], w[e].double().t().contiguous(), i),
                                    (dx[s], dy[s], w[e].double(), o)):
            want, size = rows.double() @ m, rows.double().abs() @ m.abs()
            tol = (terms + 4) * U * size
            if got.dtype == BF16:
                tol = tol + half(BF16) * (want.abs() + tol) + tiny(BF16)
            assert bool(((got.double() - want).abs() <= tol).all())
    assert bool((y[expert < 0] == 7.0).all()) and not bool(dx[expert < 0].any())
    if E == 1:  # two slots a row
        rows = x[:n // 2]
        got = ntc.linear(rows, w1, slots_per_row=2, out_dtype=F32)
        m = w[0].double().t().contiguous()
        want = (rows.double() @ m).repeat_interleave(2, 0)
        size = (rows.double().abs() @ m.abs()).repeat_interleave(2, 0)
        assert bool(((got.double() - want).abs() <= (i + 4) * U * size).all())


# -------------------------------------------------- values of mixed size


@pytest.mark.parametrize("B", [64.0, 128.0, 1000.0, 1e30])
@pytest.mark.parametrize("E,per", [(64, 2), (64, 4), (96, 3), (256, 16), (1024, 32)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_route_groups_of_cancelling_biases(dev, E, per, B, score):
    """Groups whose two best values have biases of opposite sign: their sum is near 1, its
    float32 error that of the biases' size.  Which groups stay goes by float64."""
    g = gen(int(B) % 1000 + E)
    G, n = E // per, 200
    bias = torch.full((G, per), -4 * B)
    bias[:, 0], bias[:, 1] = B, -B
    bias[1::2, :2] = 0.0  # and groups of plain scores between them
    l = torch.randn(n, G, per, generator=g)
    if score == "sigmoid":  # sums of scores a few 1e-6 apart
        first = 0.2 + 0.6 * torch.rand(n, G, generator=g).double()
        target = 0.9 + (torch.rand(n, 1, generator=g).double() - 0.5) * 0.2
        apart = torch.argsort(torch.rand(n, G, generator=g), dim=1).double() * 3e-6
        l[:, :, 0] = torch.logit(first).float()
        l[:, :, 1] = torch.logit(target + apart - torch.sigmoid(l[:, :, 0].double())).float()
    l = l.view(n, E)
    opt = dict(score=score, n_groups=G, top_groups=max(1, G // 4), group_top=2, bias=bias.view(-1))
    k = min(8, opt["top_groups"] * 2)
    ids, w = R.choose(l.double(), k, **opt)
    opt["bias"] = opt["bias"].to(dev)
    got = ntc.route(l.to(dev), k, **opt)
    assert torch.equal(got.ids.cpu(), ids)
    close(got.weights, w, (70 + E + 16) * U * w + 1e-37)


def test_route_groups_of_infinite_biases(dev):
    """+inf is a value like others: above all finite ones, equal to itself."""
    l = torch.randn(50, 64, generator=gen(3))
    for per in (2, 4, 8):
        bias = 0.1 * torch.randn(64, generator=gen(4))
        bias[[5, 40, 41]] = math.inf
        bias[[8, 9, 17]] = -math.inf
        l[::3, 40:48] = -math.inf  # a group of none, beside those of +inf
        opt = dict(score="sigmoid", n_groups=64 // per, top_groups=3, group_top=2)
        ids, _ = R.choose(l.double(), 5, bias=bias, **opt)
        assert torch.equal(ntc.route(l.to(dev), 5, bias=bias.to(dev), **opt).ids.cpu(), ids)


# --------------------------------------------------------------------- unrounded sums


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,o", [(1, 24), (300, 520), (4000, 65)])
def test_bias_gradient_sums_float32(dev, dtype, n, o):
    """The sum of dy * act'(pre) before that is rounded to the layer's type for the products."""
    g = gen(n)
    x, w = torch.zeros(n, 64, dtype=dtype, device=dev), torch.zeros(o, 64, dtype=dtype, device=dev)
    pre = torch.randn(n, o, generator=g).to(dtype)
    ids = torch.randint(0, 3, (n,), generator=g).to(torch.int32)  # experts 0 and 1, 2: none
    ids[ids == 2] = -1
    bins = ntc.build_bins(ids.to(dev), torch.arange(2, dtype=torch.int32, device=dev), 2)
    for act, from_t in (("none", F32), ("gelu", dtype), ("silu", F32), ("leaky_relu", dtype)):
        dy = torch.randn(n, o, generator=g).to(from_t)
        opt = dict(pre=None if act == "none" else pre.to(dev), activation=act,
                   leaky_slope=0.3 if act == "leaky_relu" else None, grad_dtype=F32)
        dz = dy.double() * (1.0 if act == "none" else R.act_slope(pre.double(), act, 0.3))
        off = (0.0 if act == "none" else 2.0 ** -18) * dy.double().abs() + 2 * U * dz.abs()
        one = ntc.linear_backward(dy.to(dev), x, w, **opt).bias
        each = ntc.linear_backward(dy.to(dev), x, w.expand(2, o, 64).contiguous(), bins=bins,
                                   **opt).bias
        for got, at in ((one, torch.arange(n)), (each[0], torch.nonzero(ids == 0).view(-1)),
                        (each[1], torch.nonzero(ids == 1).view(-1))):
            tol = off[at].sum(0) + (at.numel() + 2) * U * dz[at].abs().sum(0)
            close(got, dz[at].sum(0), tol)


# ----------------------------------------------------------------- arguments of the binding


def test_binding_refuses_numbers_past_32_bits(dev):
    """They would reach the library as others."""
    l, rows = torch.zeros(4, 64, device=dev), torch.zeros(8, 16, device=dev)
    x, w = torch.zeros(0, 64, dtype=BF16, device=dev), torch.zeros(8, 64, dtype=BF16, device=dev)
    ids = torch.zeros(4, 2, dtype=torch.int32, device=dev)
    wrap = 1 << 32
    calls = [lambda: ntc.route(l, 2, n_groups=wrap + 4), lambda: ntc.route(l, 2, group_top=wrap + 1),
             lambda: ntc.route(l, 2, n_groups=4, top_groups=wrap + 1),
             lambda: ntc.route(l[:0], wrap + 2),
             lambda: ntc.linear(x, w, slots_per_row=wrap + 1),
             lambda: ntc.linear_backward(x[:, :8], x, w, slots_per_row=wrap + 1),
             lambda: ntc.combine(rows[:0], k=wrap + 2),
             lambda: ntc.combine(rows, ids=ids, n_experts=wrap + 8),
             lambda: ntc.combine_backward(rows[:4], rows, ids=ids, n_experts=wrap + 8)]
    for call in calls:
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_bins_that_overlap(dev):
    """Offsets that are no binning's (each expert's bin the whole of perm) have no right
    answer; their calls stay within their buffers, and later ones are as before."""
    g = gen(7)
    n, E = 300, 24
    x, dy = torch.randn(n, 64, generator=g).to(BF16).to(dev), torch.randn(n, 96, generator=g).to(BF16).to(dev)
    w, pre = torch.randn(E, 96, 64, generator=g).to(BF16).to(dev), torch.randn(n, 96, generator=g).to(BF16).to(dev)
    ids = torch.randint(0, E, (n,), generator=g).to(torch.int32).to(dev)
    identity = torch.arange(E, dtype=torch.int32, device=dev)
    good = ntc.build_bins(ids, identity, E)
    opt = dict(pre=pre, activation="gelu")
    want = ntc.linear_backward(dy, x, w, bins=good, **opt)
    bad = ntc.build_bins(ids, identity, E)
    bad.bin_offset[0::2] = 0
    bad.bin_offset[1::2] = bad.capacity
    got = ntc.linear_backward(dy, x, w, bins=bad, **opt)
    assert got.bias.shape == (E, 96)
    got = ntc.linear_backward(dy, x, w, bins=good, **opt)
    for a, b in ((got.x, want.x), (got.weight, want.weight), (got.bias, want.bias)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("align", [1, 64])
def test_no_rows_with_bins(dev, align):
    g = gen(1)
    w = torch.randn(3, 96, 64, generator=g).to(BF16).to(dev)
    x, dy = torch.zeros(0, 64, dtype=BF16, device=dev), torch.zeros(0, 96, dtype=BF16, device=dev)
    r = ntc.route(torch.zeros(0, 3, device=dev), 2)
    assert r.ids.shape == (0, 2)
    bins = ntc.build_bins(r.ids, torch.arange(3, dtype=torch.int32, device=dev), 3, align=align)
    assert ntc.linear(x, w, bins=bins, slots_per_row=2).shape == (0, 96)
    grads = ntc.linear_backward(dy, x, w, bins=bins, slots_per_row=2)
    assert grads.x.shape == (0, 64) and not bool(grads.weight.any()) and not bool(grads.bias.any())
    assert ntc.combine(dy, r.weights, ids=r.ids, n_experts=3).shape == (0, 96)
    drows, dweights = ntc.combine_backward(dy, dy, r.weights, ids=r.ids, n_experts=3)
    assert drows.shape == (0, 96) and dweights.shape == (0, 2)
