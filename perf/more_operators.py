"""Operators that train and serve a model over the units of a network, as measurable cases: the
softmax cross entropy over many classes with its gradient, orthogonalised updates of weights, and
products of 8-bit integers.

A case is a dict of plain values:
  op        "entropy"   loss[t] = log(sum_c exp(x[t] . w[c])) - x[t] . w[targets[t]] over the valid
                        classes c, 0 for a token without a target
            "orthogonal" the orthogonalised x: with X = x / (norm(x) + eps), five times
                        X <- a X + (b A + c A A) X, A = X X^T, of the matrix or its transpose,
                        whichever is wide
            "step"      momentum <- beta momentum + gradient,
                        weights <- weights - rate scale orthogonal(gradient + beta momentum)
            "linear8"   y = (xq wq^T) xs ws, x quantised a row at a time: xs = max |x| / 127,
                        xq = x / xs rounded to nearest, ties to even
  dtype     "bf16", "f16" or "f32": the type of x, weights, gradients, results
  entropy:  tokens, dim, classes, train (the gradients of x and w too), padded (share of tokens
            without a target, whose x means nothing), shut (share of classes that are not there)
  orthogonal, step: batch (matrices), rows, cols; step: decay
  linear8:  tokens, dim, out, pad (columns of the wider buffer that x is a part of)

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
_STEPS = 5
_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
_EPS = 1e-7
_RATE, _BETA = 0.02, 0.95


def listed():
    return [
        # the log probability of one token's class: its weights are read once
        {"name": "entropy_token", "op": "entropy", "train": False, "dtype": "bf16", "tokens": 1,
         "dim": 2048, "classes": 65_536, "padded": 0.0, "shut": 0.0},
        # a serving batch scored against an odd number of classes
        {"name": "entropy_batch", "op": "entropy", "train": False, "dtype": "f16", "tokens": 64,
         "dim": 1024, "classes": 50_001, "padded": 0.0, "shut": 0.02},
        # a training step, padding at the end of the batch
        {"name": "entropy_train", "op": "entropy", "train": True, "dtype": "bf16",
         "tokens": 8_192, "dim": 2048, "classes": 131_072, "padded": 0.02, "shut": 0.0},
        # a training step of a small model in 32 bits over the units of a network, some of them
        # gone; nothing even or aligned
        {"name": "entropy_odd", "op": "entropy", "train": True, "dtype": "f32", "tokens": 1_777,
         "dim": 501, "classes": 10_007, "padded": 0.05, "shut": 0.03},
        # one small matrix: fifteen small products that wait for each other
        {"name": "orthogonal_small", "op": "orthogonal", "dtype": "f32", "batch": 1, "rows": 64,
         "cols": 192},
        # the gradients of a few experts of odd sizes, in 32 bits
        {"name": "orthogonal_odd", "op": "orthogonal", "dtype": "f32", "batch": 7, "rows": 666,
         "cols": 501},
        # an update of 64 local experts' first products
        {"name": "step_experts", "op": "step", "dtype": "bf16", "batch": 64, "rows": 2048,
         "cols": 1024, "decay": 0.01},
        # an update of a large model's layers, weights kept in 32 bits
        {"name": "step_layers", "op": "step", "dtype": "f32", "batch": 4, "rows": 2048,
         "cols": 4096, "decay": 0.01},
        # one token through a layer in 8 bits
        {"name": "linear8_token", "op": "linear8", "dtype": "bf16", "tokens": 1, "dim": 4096,
         "out": 16_384, "pad": 0},
        # a serving batch
        {"name": "linear8_batch", "op": "linear8", "dtype": "bf16", "tokens": 64, "dim": 4096,
         "out": 16_384, "pad": 0},
        # a prompt of odd length, rows cut out of a wider buffer
        {"name": "linear8_prompt", "op": "linear8", "dtype": "bf16", "tokens": 8_191,
         "dim": 4096, "out": 8192, "pad": 64},
        # nothing even or aligned
        {"name": "linear8_odd", "op": "linear8", "dtype": "f16", "tokens": 777, "dim": 501,
         "out": 1_333, "pad": 3},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width of a layer: mostly a multiple of 64, now and then any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.25 else max(64, (n + 32) // 64 * 64)


def draw(rng):
    op = rng.choice(["entropy", "entropy", "orthogonal", "step", "linear8", "linear8"])
    c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    if op == "entropy":
        c.update(train=rng.random() < 0.6, tokens=_log(rng, 1, 16_384),
                 dim=_width(rng, 64, 4096), classes=_log(rng, 100, 131_072),
                 padded=rng.choice([0.0, 0.02, 0.3]), shut=rng.choice([0.0, 0.0, 0.05]))
        most = 2.2e12 * (1 / 16 if c["dtype"] == "f32" else 1)  # products of a pass over w
        c["tokens"] = max(1, min(c["tokens"], int(most / (c["dim"] * c["classes"]))))
        return c
    if op in ("orthogonal", "step"):
        c.update(batch=_log(rng, 1, 64), rows=_width(rng, 32, 4096), cols=_width(rng, 32, 4096))
        if op == "step":
            c["decay"] = rng.choice([0.0, 0.01])
        short, long = sorted((c["rows"], c["cols"]))
        most = 1.3e11 * (1 / 2 if c["dtype"] == "f32" else 1)  # short^2 long of all matrices
        c["batch"] = max(1, min(c["batch"], int(most / (short * short * long))))
        return c
    c.update(tokens=_log(rng, 1, 16_384), dim=_width(rng, 64, 8192), out=_width(rng, 64, 16_384),
             pad=rng.choice([0, 0, 3, 64]))
    most = 2.7e11
    c["tokens"] = max(1, min(c["tokens"], int(most / (c["dim"] * c["out"]))))
    return c


def work(case):
    c = SimpleNamespace(**case)
    size = _SIZE[c.dtype]
    if c.op == "entropy":
        operands = (c.tokens + c.classes) * c.dim * size
        rows = 8 * c.tokens
        products = 2 * c.tokens * c.classes * c.dim
        if c.train:  # the logits, and the products of their gradient with w and with x
            return {"bytes": 2 * operands + rows + 4 * c.tokens, "flops": 3 * products}
        return {"bytes": operands + rows, "flops": products}
    if c.op in ("orthogonal", "step"):
        n = c.batch * c.rows * c.cols
        short, long = sorted((c.rows, c.cols))
        # A and A A are symmetric: half of each
        flops = _STEPS * c.batch * (3 * short * short * long + short ** 3)
        return {"bytes": n * (2 * size if c.op == "orthogonal" else 3 * size + 8),
                "flops": flops}
    return {"bytes": size * c.tokens * (c.dim + c.out) + c.out * (c.dim + 4),
            "flops": 2 * c.tokens * c.dim * c.out}


# ---------------------------------------------------------------------------- inputs ----

def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev, dtype = "cuda", _DTYPES[c.dtype]

    def normal(*shape, dtype=dtype, scale=1.0):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype).mul_(scale)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=dev)

    s = SimpleNamespace(c=c)
    if c.op == "entropy":
        s.w = normal(c.classes, c.dim, scale=c.dim ** -0.5)
        # some classes are met much more often than others
        often = (c.classes * uniform(c.tokens) ** 3).long().clamp(max=c.classes - 1)
        # what a model has learned so far: the target's logit stands out, here more and there less
        known = 10.0 * uniform(c.tokens, 1) ** 2
        s.x = (normal(c.tokens, c.dim, dtype=torch.float32)
               + known * s.w[often].float()).to(dtype)
        s.valid = None
        if c.shut:
            shut = uniform(c.classes) < c.shut
            shut[0] = False
            s.valid = (~shut).to(torch.uint8)
            s.w.masked_fill_(shut[:, None], math.nan)
            s.x.nan_to_num_(nan=0.5)
            often = torch.where(shut[often], 0, often)
        s.targets = often.int()
        padding = int(c.tokens * c.padded)
        if padding:
            s.targets[-padding:] = -1
            s.x[-padding:] = math.nan
        if c.train:  # a mean over the tokens, some of which count for more, and some for nothing
            weight = 0.5 + uniform(c.tokens)
            weight = weight.masked_fill(uniform(c.tokens) < 0.02, 0.0)
            scaled = 1024.0 if c.dtype == "f16" else 1.0  # (a float16 loss is scaled)
            s.dloss = weight * (scaled / c.tokens)
        return s

    if c.op in ("orthogonal", "step"):
        # gradients: a few directions much stronger than the others, and noise
        rank = min(64, c.rows, c.cols)
        strength = torch.exp(-torch.arange(rank, device=dev) / 8.0)

        def gradient(dtype, scale):
            left = normal(c.batch, c.rows, rank, dtype=torch.float32) * strength
            right = normal(c.batch, rank, c.cols, dtype=torch.float32)
            noise = normal(c.batch, c.rows, c.cols, dtype=torch.float32, scale=0.05)
            return ((torch.bmm(left, right) + noise) * scale).to(dtype)

        s.x = gradient(dtype, 1e-2)
        if c.op == "step":
            s.momentum = gradient(torch.float32, 5e-2)
            s.w = normal(c.batch, c.rows, c.cols, scale=c.cols ** -0.5)
        return s

    # activations: rows of different size, a few columns much larger than the others
    columns = torch.where(uniform(c.dim) < 0.002, 20.0, 1.0)
    size = torch.exp(0.5 * torch.randn(c.tokens, 1, generator=g, device=dev))
    x = torch.zeros(c.tokens, c.dim + c.pad, dtype=dtype, device=dev)
    x[:, :c.dim] = normal(c.tokens, c.dim, dtype=torch.float32) * columns * size
    s.x = x[:, :c.dim]
    # weights in 8 bits, as a program that serves them keeps them
    w = normal(c.out, c.dim, dtype=torch.float32, scale=c.dim ** -0.5)
    s.scales = w.abs().amax(1) / 127
    s.w = torch.round(w / s.scales[:, None]).to(torch.int8)
    return s


# ------------------------------------------------------------------------ plain form ----

def _plain_entropy(s):
    c = s.c
    there = torch.ones(c.classes, dtype=torch.bool, device=s.x.device) if s.valid is None \
        else s.valid != 0
    at = s.targets.long().clamp(0, c.classes - 1)
    live = (s.targets >= 0) & (s.targets < c.classes) & there[at]
    x = s.x.float().masked_fill(~live[:, None], 0.0)
    w = s.w.float().masked_fill(~there[:, None], 0.0)
    logits = (x @ w.t()).masked_fill(~there, -math.inf)
    top = logits.max(-1, keepdim=True)[0]
    part = torch.exp(logits - top)
    total = part.sum(-1, keepdim=True)
    chosen = logits.gather(1, at[:, None])
    loss = torch.where(live, (torch.log(total) - (chosen - top))[:, 0], 0.0)
    if not c.train:
        return {"loss": loss}
    del logits
    d = part.div_(total)
    d.scatter_add_(1, at[:, None], torch.full_like(chosen, -1.0))
    d.mul_(torch.where(live, s.dloss, 0.0)[:, None])
    return {"loss": loss, "dx": (d @ w).to(s.x.dtype), "dw": (d.t() @ x).to(s.w.dtype)}


def _plain_orthogonal(x):
    """x (batch, rows, cols) in 32 bits, orthogonalised."""
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = (x / (norm + _EPS)).float()
    a, b, c = _COEFFICIENTS
    for _ in range(_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_step(s):
    g = s.x.float()
    momentum = _BETA * s.momentum + g
    update = _plain_orthogonal(g + _BETA * momentum)
    rate = _RATE * max(1.0, s.c.rows / s.c.cols) ** 0.5
    w = s.w.float() * (1 - _RATE * s.c.decay) - rate * update
    return {"w": w.to(s.w.dtype), "momentum": momentum}


def _plain_linear8(s):
    x = s.x.float()
    scale = (x.abs().amax(1, keepdim=True) / 127).clamp(min=2.0 ** -126)
    # (values next to a border between two whole numbers)
    q = torch.round(x.double() / scale.double()).float()
    return {"y": (q @ s.w.float().t() * scale * s.scales).to(s.x.dtype)}


# --------------------------------------------------------------- the package's calls ----

def _own(s):
    from paper_1503_08294_amd import learning
    c = s.c
    if c.op == "entropy":
        if not c.train:
            return {"loss": learning.cross_entropy(s.x, s.w, s.targets, s.valid)}
        loss, lse = learning.cross_entropy_forward(s.x, s.w, s.targets, s.valid)
        dx, dw = learning.cross_entropy_backward(s.dloss, s.x, s.w, s.targets, s.valid, lse)
        return {"loss": loss, "dx": dx, "dw": dw}
    if c.op == "orthogonal":
        return {"x": learning.orthogonalise(s.x, steps=_STEPS, coefficients=_COEFFICIENTS,
                                            eps=_EPS)}
    if c.op == "step":
        w, momentum = learning.orthogonal_step(s.w, s.x, s.momentum, _RATE, beta=_BETA,
                                               decay=c.decay, steps=_STEPS,
                                               coefficients=_COEFFICIENTS, eps=_EPS)
        return {"w": w, "momentum": momentum}
    return {"y": learning.linear_8bit(s.x, s.w, s.scales)}


def run(state):
    if own:
        return _own(state)
    op = state.c.op
    if op == "entropy":
        return _plain_entropy(state)
    if op == "orthogonal":
        return {"x": _plain_orthogonal(state.x.float()).to(state.x.dtype)}
    return _plain_step(state) if op == "step" else _plain_linear8(state)


# --------------------------------------------------------------------------- 64 bits ----

def _exact_entropy(s):
    """Tokens some at a time; the gradient through log softmax's definition."""
    c = s.c
    live = s.targets >= 0  # (no target of these cases is a class that is shut)
    x = torch.where(live[:, None], s.x.double(), 0.0)
    w = s.w.double().nan_to_num(0.0)  # (of the classes that are shut alone)
    loss = torch.zeros(c.tokens, dtype=torch.float64, device=x.device)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w) if c.train else None
    for i in range(0, c.tokens, 2048):
        t = slice(i, i + 2048)
        logits = x[t] @ w.t()
        if s.valid is not None:
            logits[:, s.valid == 0] = -math.inf
        logp = torch.log_softmax(logits, -1)
        one = torch.nn.functional.one_hot(s.targets[t].long().clamp(min=0), c.classes)
        loss[t] = -torch.where(one == 1, logp, 0.0).sum(1) * live[t]
        if c.train:
            d = (logp.exp() - one) * (s.dloss[t].double() * live[t])[:, None]
            dx[t] = d @ w
            dw += d.t() @ x[t]
    return {"loss": loss, "dx": dx, "dw": dw} if c.train else {"loss": loss}


def _exact_orthogonal(x):
    """One matrix after the other, rows or columns alike: (A X) X^T = X (X^T X)."""
    out = torch.empty_like(x)
    p, q, r = _COEFFICIENTS
    for i in range(x.shape[0]):
        m = x[i] / (torch.linalg.matrix_norm(x[i]) + _EPS)
        wide = m.shape[0] <= m.shape[1]
        for _ in range(_STEPS):
            if wide:
                k = m @ m.t()
                m = p * m + (q * k + r * (k @ k)) @ m
            else:
                k = m.t() @ m
                m = p * m + m @ (q * k + r * (k @ k))
        out[i] = m
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = s.c
    if c.op == "entropy":
        return _exact_entropy(s)
    if c.op == "orthogonal":
        return {"x": _exact_orthogonal(s.x.double())}
    if c.op == "step":
        g = s.x.double()
        momentum = _BETA * s.momentum.double() + g
        update = _exact_orthogonal(g + _BETA * momentum)
        scale = math.sqrt(max(1.0, c.rows / c.cols))
        return {"w": s.w.double() - _RATE * (c.decay * s.w.double() + scale * update),
                "momentum": momentum}
    # a row's scale is held in 32 bits: the quotient by 127, rounded once
    x = s.x.double()
    scale = (x.abs().max(1, keepdim=True)[0] / 127).float().double()
    q = torch.round(x / scale)
    return {"y": (q @ s.w.double().t()) * (scale * s.scales.double())}
