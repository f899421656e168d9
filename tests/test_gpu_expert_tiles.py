"""Linear layers over bins at sizes that take the large tiles: 256 x 256 and 128 x 128 tiles
of every product, and launches whose last round is cut into smaller tiles, against float64
products on the GPU.

Beside each case stands what it is there for: `tiles` is the number of 256 x 256 tiles, of
which 256 run at once.  A last round of 1 to 128 of them is a launch of its own, in 64 x 64
tiles up to 48 and in 128 x 128 above (with bins always), where the contraction is at least
1536; the tests check these numbers, so that a case cannot lose its meaning unnoticed.

Tolerances as in test_gpu_experts.py: a sum of m float32 products in any order is off by at
most (m + 2) U times the sum S of the products' absolute values; activations multiply an error
of z by at most 1.13 and add at most 2^-19 (|z| + 1)."""
import math

import pytest
import torch

from paper_2608_27888_amd import ntc
from test_gpu_experts import BF16, F16, F32, U, dev, half, tiny  # noqa: F401 (dev: fixture)

pytestmark = pytest.mark.gpu
ROUND = 256


def up(a, b):
    return -(-a // b)


def generator(dev, seed):
    g = torch.Generator(dev)
    g.manual_seed(seed)
    return g


def padded(t, pad, fill=math.nan):
    """The matrix with `pad` more elements behind every row."""
    big = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def within(got, want, tol, to=F32):
    if to != F32:
        tol = tol + half(to) * (want.abs() + tol) + tiny(to)
    assert got.dtype == to
    off = (got.double() - want).abs() - tol
    assert bool((off <= 0).all()), off.max().item()


def slots_of(counts, outside, g, dev):
    """Expert of every slot in random order, `outside` slots of none, and their bins."""
    expert = torch.repeat_interleave(torch.arange(len(counts), device=dev),
                                     torch.tensor(counts, device=dev))
    expert = torch.cat([expert, torch.full((outside,), -1, device=dev)])
    expert = expert[torch.randperm(expert.numel(), generator=g, device=dev)].contiguous()
    bins = ntc.build_bins(expert.to(torch.int32),
                          torch.arange(len(counts), dtype=torch.int32, device=dev), len(counts))
    return expert, bins


def product(a, b):
    """(a b, |a| |b|) in float64."""
    a, b = a.double(), b.double().contiguous()
    return a @ b, a.abs() @ b.abs()


# slots, and how many tiles the last round has
@pytest.mark.parametrize("n,last", [(8400, 8), (9723, 48), (9900, 56), (12200, 128), (12300, 136),
                                    (16384, 0)])
@pytest.mark.parametrize("div", [1, 2])
def test_last_round_of_one_layer(dev, n, last, div):
    n, dim = n // div * div, 2040
    tiles = up(n, 256) * up(dim, 256)
    assert tiles > ROUND and tiles % ROUND == last and dim >= 1536
    g = generator(dev, n)
    x = torch.randn(n // div, dim, generator=g, device=dev).to(BF16)
    w = torch.randn(dim, dim, generator=g, device=dev).to(BF16)
    y = torch.full((n, dim), 7.0, device=dev)
    ntc.linear(x, w, slots_per_row=div, out=y)
    want, size = (t.repeat_interleave(div, 0) for t in product(x, w.t()))
    within(y, want, (dim + 2) * U * size)
    del want, size
    dy = torch.randn(n, dim, generator=g, device=dev).to(BF16)
    dx = ntc.linear_backward(dy, x, w, slots_per_row=div, weight_grad=False, bias_grad=False).x
    want, size = (t.view(n // div, div, dim).sum(1) for t in product(dy, w))
    within(dx, want, (dim + 2 + div) * U * size, BF16)


# slots of each expert, and how many tiles the last round has
@pytest.mark.parametrize("counts,last", [
    ([5000, 301, 3100], 24),
    ([6000, 0, 1, 255, 257, 2200], 40),
    ([8000, 4000], 128),
    ([9000, 301, 3100], 152),          # too many for a launch of their own
    ([4096, 2048, 2048, 0], 0),        # none, though the host expects some
], ids=str)
@pytest.mark.parametrize("div", [1, 2])
def test_last_round_of_experts(dev, counts, last, div):
    dim, outside = 2040, 7 + (sum(counts) + 7) % 2
    tiles = sum(up(c, 256) for c in counts) * up(dim, 256)
    assert tiles >= ROUND and tiles % ROUND == last and dim >= 1536
    g = generator(dev, len(counts))
    expert, bins = slots_of(counts, outside, g, dev)
    n = expert.numel()
    x = torch.randn(n // div, dim, generator=g, device=dev).to(F16)
    w = (torch.randn(len(counts), dim, dim, generator=g, device=dev) / 32).to(F16)
    dy = torch.randn(n, dim, generator=g, device=dev).to(F16)
    y = torch.full((n, dim), 7.0, device=dev)
    ntc.linear(x, w, bins=bins, slots_per_row=div, out=y)
    dx = ntc.linear_backward(dy, x, w, bins=bins, slots_per_row=div, weight_grad=False,
                             bias_grad=False).x
    want_dx = torch.zeros(n // div, dim, dtype=torch.float64, device=dev)
    size_dx = torch.zeros_like(want_dx)
    for e in range(len(counts)):
        at = torch.nonzero(expert == e).view(-1)
        if at.numel() == 0:
            continue
        want, size = product(x[at // div], w[e].t())
        within(y[at], want, (dim + 2) * U * size)
        want, size = product(dy[at], w[e])
        want_dx.index_add_(0, at // div, want)
        size_dx.index_add_(0, at // div, size)
    within(dx, want_dx, (dim + 2 + div) * U * size_dx, F16)
    assert bool((y[expert < 0] == 7.0).all())


WEIGHT = [
    dict(o=4104, i=2120, side=256),                     # 17 x 9 tiles of 256
    dict(o=4104, i=2120, side=256, div=2),
    dict(o=2040, i=1500, side=128),                     # 16 x 12 tiles of 128
    dict(o=2040, i=1500, side=128, div=3),
    # 8 experts of 5 x 5 tiles of 256: none, one, whole steps, parts of steps
    dict(o=1032, i=1100, side=256, counts=(0, 1, 64, 65, 500, 129, 37, 200)),
    dict(o=1032, i=1104, side=256, counts=(0, 1, 64, 65, 500, 129, 37, 200), div=2, pad=8),
    dict(o=680, i=1100, side=128, counts=(300, 0, 77)),  # 3 experts of 6 x 9 tiles of 128
]
# one layer: contractions of one step, of an odd and of an even number of steps
WEIGHT = [dict(c, n=n) for c in WEIGHT
          for n in ((sum(c["counts"]),) if "counts" in c else (6, 138, 1002))]


@pytest.mark.parametrize("c", WEIGHT, ids=str)
@pytest.mark.parametrize("dtype,grad", [(BF16, F32), (F16, F16)])
def test_weight_gradient_of_large_tiles(dev, c, dtype, grad):
    n, o, i, div, pad = c["n"], c["o"], c["i"], c.get("div", 1), c.get("pad", 0)
    counts = c.get("counts")
    E = len(counts) if counts else 1
    at_once = {64: ROUND, 128: 2 * ROUND, 256: ROUND}
    tiles = E * up(o, c["side"]) * up(i, c["side"])
    assert tiles <= at_once[c["side"]] < E * up(o, c["side"] // 2) * up(i, c["side"] // 2)
    g = generator(dev, n + o)
    if counts:
        expert, bins = slots_of(counts, 4 + n % 2, g, dev)
    else:
        expert, bins = torch.zeros(n, dtype=torch.int64, device=dev), None
    n = expert.numel()
    x = padded(torch.randn(n // div, i, generator=g, device=dev).to(dtype), pad)
    dy = padded(torch.randn(n, o, generator=g, device=dev).to(dtype), pad)
    w = torch.zeros(*([E] if counts else []), o, i, dtype=dtype, device=dev)
    got = ntc.linear_backward(dy, x, w, bins=bins, slots_per_row=div, input_grad=False,
                              grad_dtype=grad)
    for e in range(E):
        at = torch.nonzero(expert == e).view(-1)
        want, size = product(dy[at].t(), x[at // div])
        within(got.weight.view(E, o, i)[e], want, (at.numel() + 2) * U * size, grad)
        d = dy[at].double()
        within(got.bias.view(E, o)[e], d.sum(0), (at.numel() + 2) * U * d.abs().sum(0), grad)


FORWARD = [
    dict(n=4000, o=4000, side=256),                              # 16 x 16 tiles of 256
    dict(n=7500, o=4000, side=256, div=2),
    dict(n=7500, o=4000, side=256, counts=(4000, 257, 0, 3236)),
    dict(n=2000, o=1800, side=128),                              # 16 x 15 tiles of 128
    dict(n=2000, o=1800, side=128, counts=(900, 1097)),
    dict(n=130, o=700, side=64),
    dict(n=9, o=700, side=0),                                    # few rows
]


@pytest.mark.parametrize("c", FORWARD, ids=str)
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("to16", [True, False])
def test_epilogue_of_every_tile(dev, c, pad, to16):
    """Bias, pre, GELU and a residual that is the output itself, rows of several strides."""
    n, o, i, div, counts = c["n"], c["o"], 200, c.get("div", 1), c.get("counts")
    if c["side"]:
        assert up(n, 256) * up(o, 256) >= ROUND or c["side"] < 256
    dtype, to = BF16, BF16 if to16 else F32
    g = generator(dev, n + o + pad)
    E = len(counts) if counts else 1
    if counts:
        expert, bins = slots_of(counts, n - sum(counts), g, dev)
    else:
        expert, bins = torch.zeros(n, dtype=torch.int64, device=dev), None
    x = torch.randn(n // div, i, generator=g, device=dev).to(dtype)
    w = (torch.randn(E, o, i, generator=g, device=dev) * i ** -0.5).to(dtype)
    b = torch.randn(E, o, generator=g, device=dev).to(dtype)
    residual = torch.randn(n, o, generator=g, device=dev).to(to)
    y = padded(residual, pad, 5.0)
    pre = padded(torch.full((n, o), 7.0, dtype=dtype, device=dev), pad, 5.0)
    got = ntc.linear(x, w if counts else w[0], b if counts else b[0], residual=y, out=y, pre=pre,
                     activation="gelu", bins=bins, slots_per_row=div)
    assert got is y
    for e in range(E):
        at = torch.nonzero(expert == e).view(-1)
        if at.numel() == 0:
            continue
        z, size = product(x[at // div], w[e].t())
        z, size = z + b[e].double(), size + b[e].double().abs()
        off = (i + 4) * U * size
        within(pre[at], z, off, dtype)
        want = 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5))) + residual[at].double()
        within(y[at], want, 1.13 * off + 2.0 ** -19 * (z.abs() + 1) + 4 * U * want.abs(), to)
    gone = expert < 0
    assert torch.equal(y[gone], residual[gone]) and bool((pre[gone] == 7.0).all())
    if pad:  # what lies between the rows
        for t in (y, pre):
            assert bool((t.as_strided((n - 1, pad), (o + pad, 1), o) == 5.0).all())
