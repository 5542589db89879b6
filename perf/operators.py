"""The operators of a mixture of local experts, as measurable cases: layer norm, the routing of
tokens to experts, and the experts' products, each forward and, for training, backward.

A case is a dict of plain values:
  op        "norm"     y = (x - mean) * rstd * weight + bias over rows of x
            "route"    the experts of every token and their weights, from its logits
            "experts"  out[t] = sum_k weights[t, k] * w2[e] (silu(gate) * up),
                       (gate, up) = w1[e] x[t], e = ids[t, k]
  train     the backward pass too: gradients of every input that has one
  dtype     "bf16", "f16" or "f32": the type of tokens, logits and experts' weights
  norm:     rows, dim, pad (columns of the wider buffer that x is a part of), param ("f32" or
            "same": the type of weight and bias)
  route:    tokens, experts, top, score ("softmax" or "sigmoid"), balance (a bias for the
            choice), groups, top_groups, best (the best choices of a group that its score sums),
            renorm, scale
  experts:  tokens, experts, top, dim, hidden, skew (how uneven the experts' shares are),
            dropped (share of tokens that no expert gets)

With `own` false the operators are computed in their plain form, elementary torch operations in 32
bits rounded once at the end; with `own` true by the package's entry points.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_MOST = 2.4e12       # operations of a drawn case, at most
_NEAR = 1e-5         # choices nearer to each other than this are decided by rounding


def listed():
    return [
        # one token's row in a serving loop: the launch and its latency
        {"name": "norm_token", "op": "norm", "train": False, "dtype": "bf16", "rows": 1,
         "dim": 2048, "pad": 0, "param": "same"},
        # a batch of prompts, rows cut out of a wider buffer
        {"name": "norm_prompt", "op": "norm", "train": False, "dtype": "bf16", "rows": 16_384,
         "dim": 4096, "pad": 64, "param": "same"},
        # a training step at an ordinary size, weights kept in 32 bits
        {"name": "norm_train", "op": "norm", "train": True, "dtype": "bf16", "rows": 16_384,
         "dim": 2048, "pad": 0, "param": "f32"},
        # a training step in 32 bits on odd sizes: no row is aligned
        {"name": "norm_odd", "op": "norm", "train": True, "dtype": "f32", "rows": 8_191,
         "dim": 1_001, "pad": 0, "param": "f32"},
        # the experts of one token
        {"name": "route_token", "op": "route", "train": False, "dtype": "f32", "tokens": 1,
         "experts": 256, "top": 8, "score": "sigmoid", "balance": True, "groups": 8,
         "top_groups": 4, "best": 2, "renorm": True, "scale": 2.5},
        # a prompt's tokens, experts in groups and a bias for balance, padding at the end
        {"name": "route_prompt", "op": "route", "train": False, "dtype": "bf16",
         "tokens": 16_384, "experts": 256, "top": 8, "score": "sigmoid", "balance": True,
         "groups": 8, "top_groups": 4, "best": 2, "renorm": True, "scale": 2.5},
        # the largest batch of the signal sweep, softmax scores, with the logits' gradient
        {"name": "route_train", "op": "route", "train": True, "dtype": "f32",
         "tokens": 65_536, "experts": 64, "top": 2, "score": "softmax", "balance": False,
         "groups": 1, "top_groups": 1, "best": 1, "renorm": True, "scale": 1.0},
        # one token through its experts: their weights are read once
        {"name": "experts_token", "op": "experts", "train": False, "dtype": "bf16", "tokens": 1,
         "experts": 64, "top": 8, "dim": 2048, "hidden": 1024, "skew": 0.5, "dropped": 0.0},
        # a serving batch: a few tokens for every expert, all weights are read
        {"name": "experts_batch", "op": "experts", "train": False, "dtype": "f16", "tokens": 64,
         "experts": 64, "top": 8, "dim": 2048, "hidden": 1024, "skew": 0.5, "dropped": 0.02},
        # a prompt of odd length, uneven experts
        {"name": "experts_prompt", "op": "experts", "train": False, "dtype": "bf16",
         "tokens": 8_191, "experts": 64, "top": 4, "dim": 2048, "hidden": 1024, "skew": 0.5,
         "dropped": 0.01},
        # a training step
        {"name": "experts_train", "op": "experts", "train": True, "dtype": "bf16",
         "tokens": 16_384, "experts": 32, "top": 2, "dim": 2048, "hidden": 2048, "skew": 0.5,
         "dropped": 0.0},
        # a training step of a small model in 32 bits, nothing even or aligned
        {"name": "experts_odd", "op": "experts", "train": True, "dtype": "f32", "tokens": 777,
         "experts": 7, "top": 3, "dim": 501, "hidden": 333, "skew": 1.0, "dropped": 0.05},
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n - 1 if n == 3072 else n


def _width(rng, lo, hi):
    """A width of a layer: mostly a multiple of 64, now and then any number."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.25:
        return n
    n = max(64, (n + 32) // 64 * 64)
    return n - 64 if n == 3072 else n


def draw(rng):
    op = rng.choice(["norm", "norm", "route", "route", "experts", "experts", "experts"])
    c = {"op": op, "train": rng.random() < 0.5}
    if op == "norm":
        c.update(dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), rows=_log(rng, 1, 65_536),
                 dim=_width(rng, 64, 8192), pad=rng.choice([0, 0, 8, 64]),
                 param=rng.choice(["f32", "same"]))
        most = 70_000_000 // c["dim"]
        c["rows"] = min(c["rows"], most - 1 if most == 3072 else most)
        return c
    if op == "route":
        experts = rng.choice([8, 16, 32, 48, 64, 100, 128, 160, 256, 384])
        groups = rng.choice([g for g in (1, 1, 4, 8) if experts % g == 0 and experts // g >= 4])
        top_groups = max(1, groups // rng.choice([1, 2]))
        c.update(dtype=rng.choice(["f32", "bf16", "f16"]), tokens=_log(rng, 1, 65_536),
                 experts=experts, top=min(rng.choice([1, 2, 4, 6, 8]),
                                          top_groups * (experts // groups)),
                 score=rng.choice(["softmax", "sigmoid"]), balance=rng.random() < 0.5,
                 groups=groups, top_groups=top_groups, best=rng.choice([1, 2]),
                 renorm=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]))
        return c
    c.update(dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), tokens=_log(rng, 1, 16_384),
             experts=rng.choice([4, 7, 8, 16, 32, 64]), top=rng.choice([1, 2, 3, 4, 8]),
             dim=_width(rng, 128, 4096), hidden=_width(rng, 128, 2048),
             skew=rng.choice([0.0, 0.5, 1.0]), dropped=rng.choice([0.0, 0.0, 0.02]))
    c["top"] = min(c["top"], c["experts"])
    # weights of 1.2 GB at most, and no more work than the largest listed case
    while 3 * c["experts"] * c["dim"] * c["hidden"] * _SIZE[c["dtype"]] > 1_200_000_000:
        c["hidden"] = c["hidden"] // 2
    most = _MOST * (1 / 16 if c["dtype"] == "f32" else 1) / (3 if c["train"] else 1)
    most = max(1, int(most / (6 * c["top"] * c["dim"] * c["hidden"])))
    c["tokens"] = min(c["tokens"], most - 1 if most == 3072 else most)
    return c


def work(case):
    c = SimpleNamespace(**case)
    size = _SIZE[c.dtype]
    if c.op == "norm":
        n, p = c.rows * c.dim, c.dim * (4 if c.param == "f32" else size)
        if c.train:
            return {"bytes": 4 * n * size + 4 * p, "flops": 18 * n}
        return {"bytes": 2 * n * size + 2 * p, "flops": 8 * n}
    if c.op == "route":
        n = c.tokens * c.experts * size
        pairs = 8 * c.tokens * c.top
        return {"bytes": n + pairs + (n + pairs // 2 if c.train else 0),
                "flops": 8 * c.tokens * c.experts * (2 if c.train else 1)}
    rows = c.tokens * c.top
    # experts that some token goes to, were all as likely
    touched = c.experts * (1 - (1 - c.top / c.experts) ** c.tokens)
    weights = 3 * c.dim * c.hidden * size
    tokens = c.tokens * c.dim * size
    forward = {"bytes": touched * weights + 2 * tokens + 8 * rows,
               "flops": 6 * rows * c.dim * c.hidden}
    if not c.train:
        return forward
    return {"bytes": forward["bytes"] + 2 * tokens + c.experts * weights + 4 * rows,
            "flops": 3 * forward["flops"]}


# ---------------------------------------------------------------------------- inputs ----

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _choices(logits, c, balance):
    """Logits, scores and what the choice of experts goes by, in 64 bits; NaN and -inf are shut
    out."""
    l = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=torch.finfo(torch.float32).max,
                         neginf=-math.inf)
    s = torch.sigmoid(l) if c.score == "sigmoid" else torch.softmax(l, -1).nan_to_num(0.0)
    key = s if balance is None else s + balance.double()
    return l, s, key.masked_fill(l == -math.inf, -math.inf)


def _undecided(logits, c, balance):
    """Rows where the choice of a group or an expert hangs on less than 32 bits resolve."""
    _, _, key = _choices(logits, c, balance)
    rows = key.shape[0]
    near = torch.zeros(rows, dtype=torch.bool, device=key.device)
    if c.groups > 1 and c.top_groups < c.groups:
        in_group = key.view(rows, c.groups, -1)
        two = in_group.sort(-1, descending=True)[0][..., :c.best]
        value = torch.where(two == -math.inf, 0.0, two).sum(-1)
        value = torch.where(two[..., 0] == -math.inf, -math.inf, value)
        ranked, order = value.sort(-1, descending=True)
        near |= (ranked[:, c.top_groups - 1] - ranked[:, c.top_groups] < _NEAR) \
            & (ranked[:, c.top_groups] > -math.inf)
        keep = torch.zeros_like(value, dtype=torch.bool)
        keep.scatter_(1, order[:, :c.top_groups], True)
        key = in_group.masked_fill(~keep[..., None], -math.inf).view(rows, -1)
    ranked = key.sort(-1, descending=True)[0][:, :c.top + 1]
    gap = ranked[:, :-1] - ranked[:, 1:]
    return near | ((gap < _NEAR) & (ranked[:, 1:] > -math.inf)).any(-1)


def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = _generator(seed)
    dev, dtype = "cuda", _DTYPES[c.dtype]

    def normal(*shape, dtype=dtype, scale=1.0):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype).mul_(scale)

    if c.op == "norm":
        # activations of a residual stream: rows of different size, an offset, a few columns
        # much larger than the others
        columns = torch.where(torch.rand(c.dim, generator=g, device=dev) < 0.002, 20.0, 1.0)
        size = torch.exp(0.5 * torch.randn(c.rows, 1, generator=g, device=dev))
        x = torch.zeros(c.rows, c.dim + c.pad, dtype=dtype, device=dev)
        x[:, :c.dim] = (normal(c.rows, c.dim, dtype=torch.float32) + 0.1) * columns * size
        param = torch.float32 if c.param == "f32" else dtype
        s = SimpleNamespace(c=c, x=x[:, :c.dim], eps=1e-5,
                            weight=(1 + normal(c.dim, dtype=torch.float32, scale=0.1)).to(param),
                            bias=normal(c.dim, dtype=torch.float32, scale=0.1).to(param))
        s.dy = normal(c.rows, c.dim) if c.train else None
        return s

    if c.op == "route":
        offset = normal(1, c.experts, dtype=torch.float32, scale=0.5)

        def logits(rows):
            return (1.5 * normal(rows, c.experts, dtype=torch.float32) + offset).to(dtype)

        balance = None
        if c.balance:  # moved up and down in steps of a thousandth while training
            balance = torch.randint(-60, 61, (c.experts,), generator=g, device=dev) * 1e-3
            balance = balance.float()
        l = logits(c.tokens)
        # an expert that is shut out here and there
        shut = torch.rand(l.shape, generator=g, device=dev) < 0.01
        l.masked_fill_(shut, -math.inf)
        if balance is not None or (c.best > 1 and c.groups > c.top_groups):
            for _ in range(8):  # rows that rounding decides have no answer to compare: others
                bad = _undecided(l, c, balance).nonzero()[:, 0]
                if bad.numel() == 0:
                    break
                l[bad] = logits(bad.numel())
        # padding at the end of a batch: its logits mean nothing
        valid = torch.ones(c.tokens, dtype=torch.uint8, device=dev)
        padding = c.tokens // 50
        if padding:
            valid[-padding:] = 0
            l[-padding:] = math.nan
        s = SimpleNamespace(c=c, logits=l, balance=balance, valid=valid)
        s.dweights = normal(c.tokens, c.top, dtype=torch.float32) if c.train else None
        return s

    x = normal(c.tokens, c.dim)
    w1 = normal(c.experts, 2 * c.hidden, c.dim, scale=c.dim ** -0.5)
    w2 = normal(c.experts, c.dim, c.hidden, scale=c.hidden ** -0.5)
    liking = c.skew * torch.randn(1, c.experts, generator=g, device=dev)
    score, ids = (torch.randn(c.tokens, c.experts, generator=g, device=dev) + liking).topk(c.top)
    weights = torch.softmax(score, -1)
    lost = torch.rand(c.tokens, 1, generator=g, device=dev) < c.dropped
    s = SimpleNamespace(c=c, x=x, w1=w1, w2=w2, ids=ids.masked_fill(lost, -1).int().contiguous(),
                        weights=weights.masked_fill(lost, 0.0).contiguous())
    s.dout = normal(c.tokens, c.dim) if c.train else None
    return s


# ------------------------------------------------------------------------ plain form ----

def _plain_norm(s):
    x, w = s.x.float(), s.weight.float()
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(-1, keepdim=True) + s.eps)
    xn = xc * rstd
    y = (xn * w + s.bias.float()).to(s.x.dtype)
    if not s.c.train:
        return {"y": y}
    dy = s.dy.float()
    g = dy * w
    dx = rstd * (g - g.mean(-1, keepdim=True) - xn * (g * xn).mean(-1, keepdim=True))
    return {"y": y, "dx": dx.to(s.x.dtype), "dweight": (dy * xn).sum(0).to(s.weight.dtype),
            "dbias": dy.sum(0).to(s.bias.dtype)}


def _plain_route(s):
    c = s.c
    rows = c.tokens
    none = -math.inf
    l = s.logits.float()
    shut = torch.isnan(l) | (l == none) | (s.valid == 0)[:, None]
    l = l.clamp(max=torch.finfo(torch.float32).max).masked_fill(shut, none)
    if c.score == "softmax":
        top = l.max(-1, keepdim=True)[0].clamp(min=torch.finfo(torch.float32).min)
        part = torch.exp(l - top)
        score = part / part.sum(-1, keepdim=True).clamp(min=1.0)
    else:
        score = 1 / (1 + torch.exp(-l))
    choice = score if s.balance is None else score + s.balance
    choice = choice.masked_fill(shut, none)
    key = l if s.balance is None else choice  # without a bias the logits give the order
    if c.groups > 1 and c.top_groups < c.groups:
        in_group = (key if c.best == 1 else choice).view(rows, c.groups, -1)
        two = in_group.sort(-1, descending=True)[0][..., :c.best]
        value = torch.where(two == none, 0.0, two).sum(-1)
        value = torch.where(two[..., 0] == none, none, value)
        kept = value.sort(dim=-1, descending=True, stable=True)[1][:, :c.top_groups]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, kept, True)
        key = key.view(in_group.shape).masked_fill(~keep[..., None], none).view(rows, -1)
    key, ids = key.sort(dim=-1, descending=True, stable=True)
    key, ids = key[:, :c.top], ids[:, :c.top]
    missing = key == none
    chosen = score.gather(1, ids).masked_fill(missing, 0.0)
    if c.renorm:
        if c.score == "softmax":
            at = l.gather(1, ids).masked_fill(missing, none)
            most = at.max(-1, keepdim=True)[0].clamp(min=torch.finfo(torch.float32).min)
            share = torch.exp(at - most)
        else:
            share = chosen
        total = share.sum(-1, keepdim=True)
        share = torch.where(total > 0, share / total, 0.0)
    else:
        share = chosen
    weights = share * c.scale
    out = {"ids": ids.masked_fill(missing, -1).int(), "weights": weights}
    if not c.train:
        return out
    dw = s.dweights.masked_fill(missing, 0.0) * c.scale
    if c.renorm:
        back = share * (dw - (dw * share).sum(-1, keepdim=True))
        if c.score == "sigmoid":
            back = back * (1 - chosen)
        dl = torch.zeros_like(l).scatter_(1, ids, back)
    elif c.score == "sigmoid":
        dl = torch.zeros_like(l).scatter_(1, ids, dw * chosen * (1 - chosen))
    else:
        inner = (dw * chosen).sum(-1, keepdim=True)
        dl = torch.zeros_like(l).scatter_(1, ids, dw) - inner
        dl = dl * score
    out["dlogits"] = dl.masked_fill(shut, 0.0).to(s.logits.dtype)
    return out


def _plain_experts(s):
    c = s.c
    pairs = c.tokens * c.top
    x, w = s.x.float(), s.weights
    slot = s.ids.reshape(-1).long()
    token = torch.arange(pairs, device=x.device) // c.top
    live = slot >= 0
    if pairs <= c.experts and not c.train:
        # few tokens: each takes its own experts' weights
        e = slot.clamp(min=0)
        h = torch.bmm(s.w1[e].float(), x[token][:, :, None])[..., 0]
        gate, up = h[:, :c.hidden], h[:, c.hidden:]
        a = gate / (1 + torch.exp(-gate)) * up
        y = torch.bmm(s.w2[e].float(), a[:, :, None])[..., 0]
        y = torch.where(live[:, None], y, 0.0)
        out = (y.view(c.tokens, c.top, -1) * w[..., None]).sum(1)
        return {"out": out.to(s.x.dtype)}
    # every expert's rows in a buffer of the most that one expert has
    key = torch.where(live, slot, c.experts)
    order = key.sort(dim=0, stable=True)[1]
    counts = torch.bincount(key, minlength=c.experts + 1)
    room = max(1, int(counts[:c.experts].max()))
    place = torch.empty_like(slot)
    place[order] = torch.arange(pairs, device=x.device) - (counts.cumsum(0) - counts)[key[order]]
    # (pairs without an expert all share one more row at the end)
    at = torch.where(live, slot * room + place, c.experts * room)

    def spread(rows):
        full = torch.zeros(c.experts * room + 1, rows.shape[1], device=x.device)
        full[at] = rows
        return full[:-1].view(c.experts, room, -1)

    def collect(full):
        flat = full.reshape(c.experts * room, -1)
        rows = flat[at.clamp(max=c.experts * room - 1)]
        return torch.where(live[:, None], rows, 0.0)

    w1, w2 = s.w1.float(), s.w2.float()
    xe = spread(x[token])
    h = torch.bmm(xe, w1.transpose(1, 2))
    gate, up = h[..., :c.hidden], h[..., c.hidden:]
    sig = 1 / (1 + torch.exp(-gate))
    a = gate * sig * up
    y = collect(torch.bmm(a, w2.transpose(1, 2))).view(c.tokens, c.top, -1)
    out = (y * w[..., None]).sum(1).to(s.x.dtype)
    if not c.train:
        return {"out": out}
    dout = s.dout.float()
    dweights = (y * dout[:, None, :]).sum(-1)
    dy = spread(dout[token] * w.reshape(-1, 1))
    dw2 = torch.bmm(dy.transpose(1, 2), a)
    da = torch.bmm(dy, w2)
    dh = torch.cat([da * up * sig * (1 + gate * (1 - sig)), da * gate * sig], -1)
    dw1 = torch.bmm(dh.transpose(1, 2), xe)
    dx = collect(torch.bmm(dh, w1)).view(c.tokens, c.top, -1).sum(1)
    return {"out": out, "dx": dx.to(s.x.dtype), "dweights": dweights,
            "dw1": dw1.to(s.w1.dtype), "dw2": dw2.to(s.w2.dtype)}


# --------------------------------------------------------------- the package's calls ----

def _own(s):
    from paper_1503_08294_amd import mixture
    c = s.c
    if c.op == "norm":
        if not c.train:
            return {"y": mixture.layer_norm(s.x, s.weight, s.bias, s.eps)}
        y, stats = mixture.layer_norm_forward(s.x, s.weight, s.bias, s.eps)
        dx, dweight, dbias = mixture.layer_norm_backward(s.dy, s.x, s.weight, s.bias, stats)
        return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if c.op == "route":
        kw = dict(score=c.score, groups=c.groups, top_groups=c.top_groups, best=c.best,
                  renormalise=c.renorm, scale=c.scale)
        ids, weights = mixture.route(s.logits, c.top, balance=s.balance, valid=s.valid, **kw)
        if not c.train:
            return {"ids": ids, "weights": weights}
        return {"ids": ids, "weights": weights,
                "dlogits": mixture.route_backward(s.dweights, s.logits, ids, **kw)}
    if not c.train:
        return {"out": mixture.experts(s.x, s.ids, s.weights, s.w1, s.w2)}
    out, saved = mixture.experts_forward(s.x, s.ids, s.weights, s.w1, s.w2)
    dx, dweights, dw1, dw2 = mixture.experts_backward(s.dout, s.x, s.ids, s.weights, s.w1, s.w2,
                                                      saved)
    return {"out": out, "dx": dx, "dweights": dweights, "dw1": dw1, "dw2": dw2}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "route": _plain_route, "experts": _plain_experts}[state.c.op](state)


# --------------------------------------------------------------------------- 64 bits ----

def _exact_norm(s):
    x = s.x.double()
    w = s.weight.double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    std = torch.sqrt(var + s.eps)
    unit = (x - mean) / std
    out = {"y": unit * w + s.bias.double()}
    if s.c.train:
        dy = s.dy.double()
        g = dy * w
        n = x.shape[1]
        out["dx"] = (n * g - g.sum(-1, keepdim=True)
                     - unit * (g * unit).sum(-1, keepdim=True)) / (n * std)
        out["dweight"] = (dy * unit).sum(0)
        out["dbias"] = dy.sum(0)
    return out


def _exact_route(s):
    c = s.c
    l, score, choice = _choices(s.logits, c, s.balance)
    off = (s.valid == 0)[:, None]
    choice = choice.masked_fill(off, -math.inf)
    key = l.masked_fill(off, -math.inf) if s.balance is None else choice
    score = score.masked_fill(off | (l == -math.inf), 0.0)
    rows = key.shape[0]
    if c.groups > 1 and c.top_groups < c.groups:
        width = c.experts // c.groups
        by = key if c.best == 1 else choice
        best = [by[:, i * width:(i + 1) * width].topk(min(c.best, width), 1)[0]
                for i in range(c.groups)]
        value = torch.stack([torch.where(b == -math.inf, 0.0, b).sum(1)
                             .masked_fill(b[:, 0] == -math.inf, -math.inf) for b in best], 1)
        keep = torch.zeros(rows, c.groups, dtype=torch.bool, device=key.device)
        for _ in range(c.top_groups):  # the first of the largest, one at a time
            left = value.masked_fill(keep, -math.inf)
            first = (left == left.max(1, keepdim=True)[0]) & ~keep
            pick = first.to(torch.int8).argmax(1)
            keep[torch.arange(rows, device=key.device), pick] = True
        key = key.masked_fill(~keep.repeat_interleave(width, 1), -math.inf)
    ids = torch.full((rows, c.top), -1, dtype=torch.int64, device=key.device)
    for k in range(c.top):
        most = key.max(1, keepdim=True)[0]
        pick = ((key == most) & (most > -math.inf)).to(torch.int8)
        got = pick.amax(1) > 0
        at = pick.argmax(1)
        ids[:, k] = torch.where(got, at, -1)
        key = key.scatter(1, at[:, None], -math.inf)
    there = ids >= 0
    at = ids.clamp(min=0)
    p = score.gather(1, at) * there
    if c.renorm:
        if c.score == "softmax":
            le = l.gather(1, at).masked_fill(~there, -math.inf)
            share = torch.softmax(le, 1).nan_to_num(0.0)
        else:
            share = (p / p.sum(1, keepdim=True)).nan_to_num(0.0)
    else:
        share = p
    out = {"ids": ids.int(), "weights": c.scale * share}
    if c.train:
        g = c.scale * s.dweights.double() * there
        if c.renorm:  # the derivative of each chosen score's logarithm
            back = share * (g - (g * share).sum(1, keepdim=True))
            if c.score == "sigmoid":
                back = back * (1 - p)
            dl = torch.zeros_like(score).scatter_add(1, at, back * there)
        elif c.score == "sigmoid":
            dl = torch.zeros_like(score).scatter_add(1, at, g * p * (1 - p))
        else:
            ds = torch.zeros_like(score).scatter_add(1, at, g)
            dl = score * (ds - (ds * score).sum(1, keepdim=True))
        out["dlogits"] = dl
    return out


def _exact_experts(s):
    c = s.c
    x = s.x.double()
    w = s.weights.double()
    out = torch.zeros_like(x)
    if c.train:
        dout = s.dout.double()
        dx, dweights = torch.zeros_like(x), torch.zeros_like(w)
        dw1 = torch.zeros(s.w1.shape, dtype=torch.float64, device=x.device)
        dw2 = torch.zeros(s.w2.shape, dtype=torch.float64, device=x.device)
    for e in range(c.experts):
        t, k = (s.ids == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        w1, w2, xe = s.w1[e].double(), s.w2[e].double(), x[t]
        gate, up = (xe @ w1.t()).split(c.hidden, 1)
        sig = torch.sigmoid(gate)
        a = gate * sig * up
        y = a @ w2.t()
        out.index_add_(0, t, y * w[t, k][:, None])
        if c.train:
            dweights[t, k] = (y * dout[t]).sum(1)
            dy = dout[t] * w[t, k][:, None]
            dw2[e] = dy.t() @ a
            da = dy @ w2
            dgate = da * up * (sig + gate * sig * (1 - sig))
            dh = torch.cat([dgate, da * gate * sig], 1)
            dw1[e] = dh.t() @ xe
            dx.index_add_(0, t, dh @ w1)
    if not c.train:
        return {"out": out}
    return {"out": out, "dx": dx, "dweights": dweights, "dw1": dw1, "dw2": dw2}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "experts": _exact_experts}[s.c.op](s)
