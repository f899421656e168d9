"""Operators of mixtures of experts, measured: routing, linear layers (one, or one per
expert over bins) and the combination of an item's expert rows, forward and backward.

An item is sent to k of E experts by ``ntc.route``; its k slots are binned by expert with
``ntc.build_bins``, as texel queries are by decoder; ``ntc.linear`` runs every slot through
its expert's layer and ``ntc.combine`` adds an item's k rows up again.  Slot ``t * k + j`` is
item t's j-th choice; an empty slot holds the id -1.

``run`` computes an operator in elementary torch operations in 32 bits, each output rounded
once, or, with ``own``, by the library's calls.  The choice of experts is made on 64-bit
scores on both sides: the last bits of a 32-bit exponential would decide between close
experts.

Inputs are drawn on the GPU from the seed alone: items and gradients ~ N(0, 1), weights
~ N(0, 1 / in), biases ~ 0.1 N(0, 1), logits ~ 1.5 N(0, 1) plus a popularity of each expert
~ 0.5 N(0, 1), balancing biases ~ 0.05 N(0, 1).
"""
import math
from types import SimpleNamespace

import torch

DEV = "cuda"
own = False
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _route(name, op, **kw):
    c = {"name": name, "op": op, "n": 16384, "experts": 64, "k": 8, "type": "f32",
         "score": "softmax", "renorm": True, "scale": 1.0, "bias": False, "groups": 1,
         "top_groups": 1, "group_top": 1, "masked": 0.0}
    c.update(kw)
    return c


def _linear(name, op, **kw):
    c = {"name": name, "op": op, "n": 4096, "in": 4096, "out": 4096, "type": "bf16",
         "act": "none", "slope": 0.0, "bias": True, "residual": False, "rows": "same",
         "pad": 0, "grad": "same"}
    c.update(kw)
    return c


def _experts(name, op, **kw):
    c = _linear(name, op, **{"in": 2048, "out": 1024})
    c.update({"n": 4096, "experts": 64, "k": 8, "div": 8})
    c.update(kw)
    return c


def _combine(name, op, **kw):
    c = {"name": name, "op": op, "n": 8192, "k": 8, "dim": 2048, "type": "bf16",
         "residual": True, "masked": 0.0}
    c.update(kw)
    return c


def _layer(name, **kw):
    c = _route(name, "layer")
    c.update({"n": 16, "dim": 2048, "hidden": 1024, "act": "silu", "type": "bf16"})
    c.update(kw)
    return c


def listed():
    return [
        # One item while answering: a single launch's latency.
        _route("route_one", "route", n=1, k=6),
        # A prompt batch over many experts in groups, sigmoid scores with a bias that
        # balances the load, a padded tail.
        _route("route_groups", "route", experts=256, score="sigmoid", bias=True, groups=8,
               top_groups=4, group_top=2, scale=2.5, masked=0.05),
        # A training batch of odd length: the gradient of plain softmax weights, which
        # reaches every expert's logit.
        _route("route_backward", "route_backward", n=30001, experts=128, k=4, type="bf16",
               renorm=False),
        # One item through one layer while answering: the weights are read once.
        _linear("linear_token", "linear", n=1, residual=True, act="silu"),
        # A ragged batch with an odd output width, padded rows, float rows out.
        _linear("linear_ragged", "linear", n=777, out=1533, type="f16", act="gelu", rows="f32",
                pad=8, **{"in": 1000}),
        # The largest: a long batch through a wide layer.
        _linear("linear_large", "linear", n=16384, out=8192, act="gelu", residual=False),
        # The gradients of such a layer at half the size: input, weight and bias.
        _linear("linear_backward", "linear_backward", n=8192, act="gelu"),
        # A prompt batch through the experts' first layer, loads uneven.
        _experts("experts_prefill", "linear"),
        # A training batch through few larger experts, float gradients of the weights.
        _experts("experts_backward", "linear_backward", n=8000, experts=8, k=2, div=2,
                 type="f16", act="relu", grad="f32", out=4096),
        # An item's rows brought together with the residual stream, prompt batch.
        _combine("combine_large", "combine"),
        # The gradients of it in training, odd sizes.
        _combine("combine_backward", "combine_backward", n=8191, k=4, dim=2056, type="f16"),
        # The whole of it for a few items while answering: routing, binning, both
        # layers, combination.
        _layer("layer_few"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_route(rng, c, most):
    c["n"] = _log_int(rng, 1, most)
    c["experts"] = rng.choice([8, 16, 40, 60, 64, 96, 128, 160, 256, 256])
    c["k"] = rng.randint(1, min(8, c["experts"]))
    c["type"] = rng.choice(["f32", "f32", "bf16", "f16"])
    c["score"] = rng.choice(["softmax", "sigmoid"])
    c["renorm"] = rng.random() < 0.6
    c["scale"] = rng.choice([1.0, 1.0, 2.5])
    c["bias"] = rng.random() < 0.4
    c["masked"] = rng.choice([0.0, 0.0, 0.1])
    if c["experts"] >= 40 and rng.random() < 0.5:
        c["groups"] = rng.choice([4, 8])
        c["top_groups"] = rng.randint(1, c["groups"])
        c["group_top"] = rng.choice([1, 2])
        c["k"] = min(c["k"], c["top_groups"] * (c["experts"] // c["groups"]))
    return c


def draw(rng):
    op = rng.choice(["route", "route", "route_backward", "linear", "linear", "linear_backward",
                     "experts", "experts", "experts_backward", "combine", "combine_backward",
                     "layer"])
    if op in ("route", "route_backward"):
        c = _draw_route(rng, _route("", op), 1 << 15)
    elif op in ("combine", "combine_backward"):
        c = _combine("", op, n=_log_int(rng, 1, 8192), k=rng.randint(1, 8),
                     dim=_log_int(rng, 64, 2048), type=rng.choice(["bf16", "f16", "f32"]),
                     residual=rng.random() < 0.5, masked=rng.choice([0.0, 0.1]))
        if rng.random() < 0.5:
            c["dim"] = (c["dim"] + 7) // 8 * 8
        if op == "combine_backward" or c["type"] == "f32":
            c["n"] = min(c["n"], 4096)
    elif op == "layer":
        c = _draw_route(rng, _layer("", n=1), 256)
        c["type"] = rng.choice(["bf16", "f16"])
        c["dim"] = rng.choice([512, 1000, 1024, 2048])
        c["hidden"] = rng.choice([256, 520, 1024])
        c["act"] = rng.choice(["relu", "gelu", "silu"])
        c["experts"] = min(c["experts"], 128)
        c["groups"], c["top_groups"], c["group_top"] = 1, 1, 1
        c["k"] = min(c["k"], c["experts"])
    else:
        experts = op.startswith("experts")
        back = op.endswith("backward")
        c = (_experts if experts else _linear)("", "linear_backward" if back else "linear")
        c["n"] = _log_int(rng, 16 if back else 1, 4096 if experts or back else 16384)
        c["in"] = _log_int(rng, 64, 4096)
        c["out"] = _log_int(rng, 64, 4096)
        if rng.random() < 0.7:  # the usual multiples
            c["in"], c["out"] = ((v + 63) // 64 * 64 for v in (c["in"], c["out"]))
        c["type"] = rng.choice(["bf16", "f16"])
        c["act"] = rng.choice(["none", "relu", "leaky_relu", "gelu", "silu"])
        c["slope"] = 0.01 if c["act"] == "leaky_relu" else 0.0
        c["bias"] = rng.random() < 0.7
        c["pad"] = rng.choice([0, 0, 8, 3])
        if back:
            # Float gradients where the activation's derivative is 0 or 1: elsewhere the
            # layer's 16-bit type rounds what flows back, and they would not be finer.
            c["grad"] = rng.choice(["same", "f32"]) if c["act"] in ("none", "relu") else "same"
        else:
            c["residual"] = rng.random() < 0.4
            c["rows"] = rng.choice(["same", "same", "f32"])
        if experts:
            c["experts"] = _log_int(rng, 2, 128)
            c["k"] = rng.randint(1, min(8, c["experts"]))
            c["div"] = rng.choice([c["k"], 1])
            c["in"], c["out"] = min(c["in"], 2048), min(c["out"], 2048)
    del c["name"]
    return c


# ------------------------------------------------------------------------------- inputs


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    t = torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)
    return t.mul_(scale).to(dtype)


def _rows(g, n, dim, dtype, pad):
    """n rows of dim values, `pad` more between one row and the next."""
    return _normal(g, n, dim + pad, dtype=dtype)[:, :dim]


def _logits(g, n, experts):
    return _normal(g, n, experts, scale=1.5) + _normal(g, experts, scale=0.5)


def _chosen(g, n, experts, k):
    """k distinct experts of every item, the popular ones more often."""
    return torch.topk(_logits(g, n, experts), k, dim=1).indices.to(torch.int32).contiguous()


def _mask(g, n, share):
    """Items that count: the last ones are padding."""
    if share == 0.0:
        return None
    mask = torch.ones(n, dtype=torch.bool, device=DEV)
    mask[n - int(share * n):] = False
    return mask


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    c = SimpleNamespace(**{("in_dim" if k == "in" else "out_dim" if k == "out" else k): v
                           for k, v in case.items()})
    s = SimpleNamespace(c=c)
    if c.op in ("route", "route_backward", "layer"):
        s.logits = _logits(g, c.n, c.experts).to(TYPES["f32" if c.op == "layer" else c.type])
        s.bias = _normal(g, c.experts, scale=0.05) if c.bias else None
        s.mask = _mask(g, c.n, c.masked)
        if c.op == "route_backward":
            s.ids = _choose(s.logits, c, s.bias, s.mask)
            s.dweights = _normal(g, c.n, c.k)
        if c.op == "layer":
            t = TYPES[c.type]
            s.x = _normal(g, c.n, c.dim, dtype=t)
            s.w1 = _normal(g, c.experts, c.hidden, c.dim, dtype=t, scale=c.dim ** -0.5)
            s.b1 = _normal(g, c.experts, c.hidden, dtype=t, scale=0.1)
            s.w2 = _normal(g, c.experts, c.dim, c.hidden, dtype=t, scale=c.hidden ** -0.5)
            s.b2 = _normal(g, c.experts, c.dim, dtype=t, scale=0.1)
            s.identity = torch.arange(c.experts, dtype=torch.int32, device=DEV)
        return s
    t = TYPES[c.type]
    if c.op in ("combine", "combine_backward"):
        s.experts = 64
        s.ids = _chosen(g, c.n, s.experts, c.k)
        mask = _mask(g, c.n, c.masked)
        s.weights = torch.softmax(_normal(g, c.n, c.k), 1)
        if mask is not None:
            s.ids[~mask] = -1
            s.weights[~mask] = 0.0
        s.rows = _normal(g, c.n * c.k, c.dim, dtype=t)
        s.residual = _normal(g, c.n, c.dim, dtype=t) if c.residual else None
        s.dout = _normal(g, c.n, c.dim, dtype=t) if c.op == "combine_backward" else None
        return s
    # a linear layer, or the experts' layers over the slots
    grouped = hasattr(c, "experts")
    s.ids, s.identity, shape, slots, s.div = None, None, (), c.n, 1
    if grouped:
        s.ids = _chosen(g, c.n, c.experts, c.k)
        s.identity = torch.arange(c.experts, dtype=torch.int32, device=DEV)
        shape, slots, s.div = (c.experts,), c.n * c.k, c.div
    s.slots = slots
    s.x = _rows(g, slots // s.div, c.in_dim, t, c.pad)
    s.weight = _normal(g, *shape, c.out_dim, c.in_dim, dtype=t, scale=c.in_dim ** -0.5)
    s.bias = _normal(g, *shape, c.out_dim, dtype=t, scale=0.1) if c.bias else None
    if c.op == "linear":
        to = TYPES["f32"] if c.rows == "f32" else t
        s.residual = _rows(g, slots, c.out_dim, to, c.pad) if c.residual else None
    else:
        s.dy = _rows(g, slots, c.out_dim, t, c.pad)
        s.pre = None
        if c.act != "none":  # what the forward pass kept
            s.pre = torch.empty(slots, c.out_dim, dtype=t, device=DEV)
            for rows, w, b in _per_expert(s):
                z = s.x[rows // s.div].float() @ w.float().t()
                s.pre[rows] = (z if b is None else z + b.float()).to(t)
    return s


# --------------------------------------------------------------------------- plain forms


def _scores(l, score):
    """64-bit scores of the logits; experts that cannot be chosen score 0."""
    l = l.double()
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    e = torch.exp(l - l.max(1, keepdim=True).values)
    return e / e.sum(1, keepdim=True)


def _choose(logits, c, bias, mask):
    """The k experts of every item: int32 [n][k], -1 past the eligible ones."""
    n, E = logits.shape
    s = _scores(logits, c.score)
    value = logits.double() if bias is None else s + bias.double()
    gone = torch.isnan(logits) | (logits.double() == -math.inf)
    if mask is not None:
        gone = gone | ~mask[:, None]
    value = value.masked_fill(gone, -math.inf)
    if c.groups > 1:
        per = value.view(n, c.groups, -1)
        if c.group_top == 1:
            best = per.max(2).values
        else:
            two = (s if bias is None else value).masked_fill(gone, -math.inf)
            two = torch.sort(two.view(n, c.groups, -1), dim=2, descending=True).values[..., :2]
            best = torch.where(two == -math.inf, torch.zeros_like(two), two).sum(2)
            best = torch.where(two[..., 0] == -math.inf, two[..., 0], best)
        order = torch.sort(best, dim=1, descending=True, stable=True).indices
        keep = torch.zeros(n, c.groups, dtype=torch.bool, device=logits.device)
        keep.scatter_(1, order[:, :c.top_groups], True)
        value = value.masked_fill(~keep.repeat_interleave(E // c.groups, 1), -math.inf)
    best, ids = torch.sort(value, dim=1, descending=True, stable=True)
    best, ids = best[:, :c.k], ids[:, :c.k]
    return torch.where(best == -math.inf, torch.full_like(ids, -1), ids).to(torch.int32)


def _shares(logits, ids, c):
    """(scores of the chosen, their weights before the scale), 32 bits; 0 at empty slots."""
    l = logits.float()
    at = l.gather(1, ids.clamp(min=0).long())
    at = at.masked_fill(ids < 0, -math.inf)
    if c.score == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-at))
        p = s / s.sum(1, keepdim=True) if c.renorm else s
    else:
        top = l.max(1, keepdim=True).values
        s = torch.exp(at - top) / torch.exp(l - top).sum(1, keepdim=True)
        p = s
        if c.renorm:
            e = torch.exp(at - at.max(1, keepdim=True).values)
            p = e / e.sum(1, keepdim=True)
    return s, torch.where(ids < 0, torch.zeros_like(p), p)


def _route_plain(s):
    ids = _choose(s.logits, s.c, s.bias, s.mask)
    return ids, _shares(s.logits, ids, s.c)[1] * s.c.scale


def _route_backward_plain(s):
    c = s.c
    score, p = _shares(s.logits, s.ids, c)
    g = torch.where(s.ids < 0, torch.zeros_like(s.dweights), s.dweights)
    l = s.logits.float()
    if c.renorm:
        d = p * (g - (p * g).sum(1, keepdim=True))
        if c.score == "sigmoid":
            d = d * (1.0 - score)
    elif c.score == "sigmoid":
        d = g * score * (1.0 - score)
    else:
        d = p * g
    d = torch.where(s.ids < 0, torch.zeros_like(d), d)
    out = torch.zeros_like(l).scatter_add_(1, s.ids.clamp(min=0).long(), d)
    if c.score == "softmax" and not c.renorm:
        e = torch.exp(l - l.max(1, keepdim=True).values)
        out = out - e / e.sum(1, keepdim=True) * (p * g).sum(1, keepdim=True)
    return (out * c.scale).to(s.logits.dtype)


def _activate(z, act, slope):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "leaky_relu":
        return torch.maximum(z, slope * z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope_at(z, act, slope):
    """The activation's derivative."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "leaky_relu":
        return torch.where(z > 0, torch.ones_like(z), torch.full_like(z, slope))
    if act == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5)
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return t * (1.0 + z * (1.0 - t))
    return torch.ones_like(z)


def _per_expert(s):
    """(slots, weight, bias) of every expert that has any; one dense layer has all rows."""
    if s.ids is None:
        yield torch.arange(s.slots, device=DEV), s.weight, s.bias
        return
    flat = s.ids.view(-1).long()
    order = torch.sort(flat, stable=True).indices
    counts = torch.bincount(flat, minlength=s.c.experts).tolist()
    at = 0
    for e, count in enumerate(counts):
        if count:
            yield order[at:at + count], s.weight[e], None if s.bias is None else s.bias[e]
        at += count


def _linear_plain(s):
    c = s.c
    t = TYPES["f32"] if c.rows == "f32" else s.x.dtype
    y = torch.empty(s.slots, c.out_dim, dtype=t, device=DEV)
    for rows, w, b in _per_expert(s):
        z = s.x[rows // s.div].float() @ w.float().t()
        z = _activate(z if b is None else z + b.float(), c.act, c.slope)
        y[rows] = (z if s.residual is None else z + s.residual[rows].float()).to(t)
    return y


def _linear_backward_plain(s):
    c = s.c
    t = s.x.dtype
    grad = TYPES["f32"] if c.grad == "f32" else t
    dx = torch.zeros(s.x.shape[0], c.in_dim, device=DEV)
    dw = torch.zeros(s.weight.shape, dtype=grad, device=DEV)
    db = torch.zeros(s.weight.shape[:-1], dtype=grad, device=DEV) if c.bias else None
    flat = None if s.ids is None else s.ids.view(-1)
    for rows, w, _ in _per_expert(s):
        dz = s.dy[rows].float()
        if s.pre is not None:
            dz = dz * _slope_at(s.pre[rows].float(), c.act, c.slope)
        dx.index_add_(0, rows // s.div, dz @ w.float())
        dwe = (dz.t() @ s.x[rows // s.div].float()).to(grad)
        if flat is None:
            dw, at = dwe, None
        else:
            at = flat[rows[0]].long()
            dw[at] = dwe
        if db is not None:
            if at is None:
                db = dz.sum(0).to(grad)
            else:
                db[at] = dz.sum(0).to(grad)
    return [dx.to(t), dw] + ([db] if c.bias else [])


def _combine_plain(rows, weights, ids, residual):
    n, k = weights.shape
    r = rows.float().view(n, k, -1)
    r = torch.where((ids < 0)[..., None], torch.zeros_like(r), r * weights[..., None])
    out = r.sum(1)
    return (out if residual is None else out + residual.float()).to(rows.dtype)


def _combine_backward_plain(s):
    n, k = s.weights.shape
    gone = (s.ids < 0)[..., None]
    d = s.dout.float()[:, None, :]
    drows = torch.where(gone, torch.zeros_like(d), s.weights[..., None] * d)
    r = s.rows.float().view(n, k, -1)
    dweights = torch.where(gone, torch.zeros_like(r), r * d).sum(2)
    return [drows.view(n * k, -1).to(s.rows.dtype), dweights]


def _layer_plain(s):
    c = s.c
    ids, weights = _route_plain(s)
    out = s.x.float()
    for e in range(c.experts):
        item, slot = torch.nonzero(ids == e, as_tuple=True)
        if item.numel() == 0:
            continue
        h = s.x[item].float() @ s.w1[e].float().t() + s.b1[e].float()
        y = _activate(h, c.act, 0.0) @ s.w2[e].float().t() + s.b2[e].float()
        out = out.index_add(0, item, y * weights[item, slot][:, None])
    return [out.to(s.x.dtype), ids, weights]


# ------------------------------------------------------------------------- the library's


def _bins(ntc, ids, identity):
    """Slots by expert, as queries by decoder."""
    return ntc.build_bins(ids.view(-1), identity, identity.numel())


def _routes(ntc, s):
    c = s.c
    return ntc.route(s.logits, c.k, score=c.score, bias=s.bias, n_groups=c.groups,
                     top_groups=c.top_groups, group_top=c.group_top, renormalize=c.renorm,
                     scale=c.scale, mask=s.mask)


def _run_own(s):
    from paper_2608_27888_amd import ntc

    c = s.c
    if c.op == "route":
        r = _routes(ntc, s)
        return [r.ids, r.weights]
    if c.op == "route_backward":
        return ntc.route_backward(s.logits, s.ids, s.dweights, score=c.score,
                                  renormalize=c.renorm, scale=c.scale)
    if c.op == "linear":
        bins = None if s.ids is None else _bins(ntc, s.ids, s.identity)
        return ntc.linear(s.x, s.weight, s.bias, residual=s.residual, activation=c.act,
                          leaky_slope=c.slope or None, bins=bins, slots_per_row=s.div,
                          out_dtype=torch.float32 if c.rows == "f32" else None)
    if c.op == "linear_backward":
        bins = None if s.ids is None else _bins(ntc, s.ids, s.identity)
        g = ntc.linear_backward(s.dy, s.x, s.weight, pre=s.pre, activation=c.act,
                                leaky_slope=c.slope or None, bins=bins, slots_per_row=s.div,
                                bias_grad=c.bias,
                                grad_dtype=torch.float32 if c.grad == "f32" else None)
        return [g.x, g.weight] + ([g.bias] if c.bias else [])
    if c.op == "combine":
        return ntc.combine(s.rows, s.weights, ids=s.ids, n_experts=s.experts,
                           residual=s.residual)
    if c.op == "combine_backward":
        return list(ntc.combine_backward(s.dout, s.rows, s.weights, ids=s.ids,
                                         n_experts=s.experts))
    r = _routes(ntc, s)
    bins = _bins(ntc, r.ids, s.identity)
    h = ntc.linear(s.x, s.w1, s.b1, activation=c.act, bins=bins, slots_per_row=c.k)
    y = ntc.linear(h, s.w2, s.b2, bins=bins)
    out = ntc.combine(y, r.weights, ids=r.ids, n_experts=c.experts, residual=s.x)
    return [out, r.ids, r.weights]


def run(s):
    if own:
        return _run_own(s)
    op = s.c.op
    if op == "route":
        return list(_route_plain(s))
    if op == "route_backward":
        return _route_backward_plain(s)
    if op == "linear":
        return _linear_plain(s)
    if op == "linear_backward":
        return _linear_backward_plain(s)
    if op == "combine":
        return _combine_plain(s.rows, s.weights, s.ids, s.residual)
    if op == "combine_backward":
        return _combine_backward_plain(s)
    return _layer_plain(s)


# ---------------------------------------------------------------------------------- work


def work(case):
    c = case
    size = {"f16": 2, "bf16": 2, "f32": 4}[c["type"]]
    if c["op"] in ("route", "route_backward"):
        n, E, k = c["n"], c["experts"], c["k"]
        if c["op"] == "route":
            b = n * E * size + n * k * 8 + (n if c["masked"] else 0) + (E * 4 if c["bias"] else 0)
        else:
            b = 2 * n * E * size + n * k * 8
        return {"bytes": b, "flops": 10 * n * E}
    if c["op"] in ("combine", "combine_backward"):
        n, k, d = c["n"], c["k"], c["dim"]
        if c["op"] == "combine":
            b = n * k * d * size + n * d * size * (2 if c["residual"] else 1) + n * k * 8
        else:
            b = 2 * n * k * d * size + n * d * size + n * k * 12
        return {"bytes": b, "flops": (2 if c["op"] == "combine" else 3) * n * k * d}
    if c["op"] == "layer":
        slots, d, f = c["n"] * c["k"], c["dim"], c["hidden"]
        b = min(c["experts"], slots) * (2 * d * f + d + f) * size
        b += c["n"] * (2 * d * size + c["experts"] * 4 + c["k"] * 8)
        return {"bytes": b, "flops": 4 * slots * d * f}
    slots = c["n"] * c.get("k", 1)
    weights = min(c.get("experts", 1), slots) * c["in"] * c["out"]
    items = slots // c.get("div", 1)
    if c["op"] == "linear":
        to = 4 if c["rows"] == "f32" else size
        b = weights * size + items * c["in"] * size + slots * c["out"] * to
        b += slots * c["out"] * to if c["residual"] else 0
        return {"bytes": b, "flops": 2 * slots * c["in"] * c["out"]}
    grads = c.get("experts", 1) * c["in"] * c["out"] * (4 if c["grad"] == "f32" else size)
    b = weights * size + grads + 2 * items * c["in"] * size
    b += slots * c["out"] * size * (1 if c["act"] == "none" else 2)
    return {"bytes": b, "flops": 4 * slots * c["in"] * c["out"]}


# ------------------------------------------------------------------- from the definition


def _exact_act(z, act, slope):
    return {"none": lambda: z, "relu": lambda: z * (z > 0),
            "leaky_relu": lambda: z * torch.where(z > 0, 1.0, slope),
            "gelu": lambda: z * torch.special.ndtr(z),
            "silu": lambda: z * torch.sigmoid(z)}[act]()


def _exact_slope(z, act, slope):
    if act in ("none", "relu", "leaky_relu"):
        return torch.where(z > 0, 1.0, {"none": 1.0, "relu": 0.0, "leaky_relu": slope}[act])
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)


def _exact_route(s, c):
    """Round by round: the best expert that is left, of the groups that are kept."""
    l = s.logits.double()
    n, E = l.shape
    f = torch.softmax(l, 1) if c.score == "softmax" else torch.sigmoid(l)
    v = l.clone() if s.bias is None else f + s.bias.double()
    if c.groups > 1:
        of = lambda t: t.reshape(n, c.groups, E // c.groups)
        if c.group_top == 1:
            best = of(v).amax(2)
        else:
            best = torch.topk(of(f if s.bias is None else v), 2, dim=2).values.sum(2)
        keep = torch.zeros(n, c.groups, dtype=torch.bool, device=l.device)
        for _ in range(c.top_groups):
            top = best.amax(1, keepdim=True)
            first = torch.argmax((best == top).to(torch.int32), 1, keepdim=True)
            keep.scatter_(1, first, True)
            best = best.scatter(1, first, -math.inf)
        v = torch.where(keep.repeat_interleave(E // c.groups, 1), v, -math.inf)
    ids = []
    for _ in range(c.k):
        top = v.amax(1, keepdim=True)
        ids.append(torch.argmax((v == top).to(torch.int32), 1, keepdim=True))
        v = v.scatter(1, ids[-1], -math.inf)
    ids = torch.cat(ids, 1)
    w = f.gather(1, ids)
    if c.renorm:
        w = w / w.sum(1, keepdim=True)
    w = w * c.scale
    if s.mask is not None:
        ids, w = torch.where(s.mask[:, None], ids, -1), torch.where(s.mask[:, None], w, 0.0)
    return ids, w


def _exact_route_backward(s, c):
    """Through the weights' Jacobian, by automatic differentiation."""
    l = s.logits.double().requires_grad_(True)
    f = torch.softmax(l, 1) if c.score == "softmax" else torch.sigmoid(l)
    live = s.ids >= 0
    w = torch.where(live, f.gather(1, s.ids.clamp(min=0).long()), 0.0)
    if c.renorm:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    (w * c.scale * torch.where(live, s.dweights.double(), 0.0)).sum().backward()
    return l.grad


def exact(case, seed):
    s = prepare(case, seed)
    c = s.c
    if c.op == "route":
        ids, w = _exact_route(s, c)
        return [ids.to(torch.int32), w]
    if c.op == "route_backward":
        return _exact_route_backward(s, c)
    if c.op == "combine":
        out = torch.zeros(c.n, c.dim, dtype=torch.float64, device=DEV)
        for j in range(c.k):
            row = s.rows[j::c.k].double() * s.weights[:, j:j + 1].double()
            out += torch.where(s.ids[:, j:j + 1] < 0, 0.0, row)
        return out if s.residual is None else out + s.residual.double()
    if c.op == "combine_backward":
        drows = torch.zeros(c.n * c.k, c.dim, dtype=torch.float64, device=DEV)
        dweights = torch.zeros(c.n, c.k, dtype=torch.float64, device=DEV)
        d = s.dout.double()
        for j in range(c.k):
            live = (s.ids[:, j:j + 1] >= 0).double()
            drows[j::c.k] = d * s.weights[:, j:j + 1].double() * live
            dweights[:, j] = (d * s.rows[j::c.k].double() * live).sum(1)
        return [drows, dweights]
    if c.op == "layer":
        ids, w = _exact_route(s, c)
        out = s.x.double()
        for e in range(c.experts):
            hit = (ids == e)
            t = torch.nonzero(hit.any(1)).view(-1)
            if t.numel():
                a = _exact_act(s.x[t].double() @ s.w1[e].double().t() + s.b1[e].double(),
                               c.act, 0.0)
                y = a @ s.w2[e].double().t() + s.b2[e].double()
                out[t] += y * (w * hit)[t].sum(1, keepdim=True)
        return [out, ids.to(torch.int32), w]
    W = s.weight.double().reshape(-1, c.out_dim, c.in_dim)
    B = None if s.bias is None else s.bias.double().reshape(-1, c.out_dim)
    expert = (torch.zeros(s.slots, dtype=torch.int64, device=DEV) if s.ids is None
              else s.ids.reshape(-1).long())
    x = s.x.double()
    item = torch.arange(s.slots, device=DEV) // s.div
    if c.op == "linear":
        y = torch.zeros(s.slots, c.out_dim, dtype=torch.float64, device=DEV)
        for e in range(W.shape[0]):
            at = torch.nonzero(expert == e).view(-1)
            z = x[item[at]] @ W[e].t()
            y[at] = _exact_act(z if B is None else z + B[e], c.act, c.slope)
        return y if s.residual is None else y + s.residual.double()
    dz = s.dy.double()
    if s.pre is not None:
        dz = dz * _exact_slope(s.pre.double(), c.act, c.slope)
    dx, dW = torch.zeros_like(x), torch.zeros_like(W)
    dB = torch.zeros(W.shape[:2], dtype=torch.float64, device=DEV)
    for e in range(W.shape[0]):
        at = torch.nonzero(expert == e).view(-1)
        dx.index_add_(0, item[at], dz[at] @ W[e])
        dW[e] = dz[at].t() @ x[item[at]]
        dB[e] = dz[at].sum(0)
    return [dx, dW.reshape(s.weight.shape)] + ([dB.reshape(s.weight.shape[:-1])] if c.bias else [])
