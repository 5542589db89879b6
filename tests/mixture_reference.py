"""Plain 64-bit definitions of the mixture's operators (numpy and torch on the CPU), written
token by token, for the tests to compare with."""
import math

import numpy as np
import torch

# the largest relative error of one rounding to the type
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def layer_norm(x, w, b, eps, dy=None):
    """y, or (y, dx, dw, db), in float64."""
    x = x.double()
    d = x.shape[1]
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    r = 1 / torch.sqrt((xc * xc).mean(1, keepdim=True) + eps)
    n = xc * r
    one = torch.ones(d, dtype=torch.float64)
    wd = one if w is None else w.double()
    y = n * wd + (0 if b is None else b.double())
    if dy is None:
        return y
    dy = dy.double()
    g = dy * wd
    dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    return y, dx, (dy * n).sum(0), dy.sum(0)


def scores(logits, score):
    l = np.where(np.isnan(logits), -np.inf, np.minimum(logits, np.finfo(np.float32).max))
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return l, 1 / (1 + np.exp(-l))
    top = max(l.max(), -np.finfo(np.float32).max)
    p = np.exp(l - top)
    return l, p / p.sum() if p.sum() > 0 else p


def route_token(logits, k, score, balance, groups, top_groups, best, renorm, scale, valid):
    """(ids, weights) of one token's float64 logits."""
    e = len(logits)
    l, s = scores(np.asarray(logits, np.float64), score)
    c = s if balance is None else s + balance
    key = l if balance is None else c
    open_ = [i for i in range(e) if valid and l[i] > -np.inf and key[i] > -np.inf]
    if groups > 1 and top_groups < groups:
        width = e // groups
        value = {}
        for i in open_:
            value.setdefault(i // width, []).append(i)
        for g, members in value.items():
            two = sorted(members, key=lambda i: (-key[i], i))[:2]
            value[g] = key[two[0]] if best == 1 else sum(c[i] for i in two)
        kept = sorted(value, key=lambda g: (-value[g], g))[:top_groups]
        open_ = [i for i in open_ if i // width in kept]
    chosen = sorted(open_, key=lambda i: (-key[i], i))[:k]
    w = share(l, s, chosen, score, renorm)
    ids = chosen + [-1] * (k - len(chosen))
    return ids, [scale * v for v in w] + [0.0] * (k - len(chosen))


def share(l, s, chosen, score, renorm):
    if not renorm or not chosen:
        return [s[i] for i in chosen]
    if score == "softmax":
        p = np.exp(l[chosen] - l[chosen].max())
    else:  # log-sigmoid, so that a set of tiny scores keeps its shares
        ls = np.array([-math.log1p(math.exp(-v)) if v > 0 else v - math.log1p(math.exp(v))
                       for v in l[chosen]])
        p = np.exp(ls - ls.max())
    return list(p / p.sum())


def route_weights(logits, ids, score, renorm, scale):
    """Differentiable weights of given ids (float64 torch tensors), 0 for -1."""
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    there = ids >= 0
    at = ids.clamp(min=0).long()
    if renorm:
        ls = l if score == "softmax" else torch.nn.functional.logsigmoid(l)
        z = ls.gather(1, at).masked_fill(~there, -1e300)
        w = torch.softmax(z, 1)
    else:
        w = (torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)).gather(1, at)
    return torch.where(there, w, torch.zeros_like(w)) * scale


def experts(x, ids, weights, w1, w2):
    """out in float64 (differentiable), one pair after another."""
    e, d, f = w2.shape
    rows = []
    for t in range(x.shape[0]):
        y = torch.zeros(d, dtype=torch.float64)
        for k in range(ids.shape[1]):
            i = int(ids[t, k])
            if 0 <= i < e:
                h = w1[i] @ x[t]
                y = y + weights[t, k] * (w2[i] @ (torch.nn.functional.silu(h[:f]) * h[f:]))
        rows.append(y)
    return torch.stack(rows) if rows else torch.zeros((0, d), dtype=torch.float64)
