"""Local experts on torch tensors: layer norm, routing of tokens to experts, and the experts'
products, through the C calls of ``include/gsn.h``.

A network of units answers with the nearest units of a signal; a mixture of local experts
answers with what the models of its best units say about it.  ``route`` picks every token's
experts (of the negative squared distances to the units with ``top=2``: the winner and the
second of ``Network.find_winners``), ``experts`` runs their products, ``layer_norm`` goes before
them.  ``layer_norm``, ``route`` and ``experts`` take part in autograd, once: derivatives of their
gradients raise ``RuntimeError``, and tensors that carry a forward-mode tangent are refused.  The
``_forward`` and ``_backward`` calls are their two halves for programs that keep their own order.

Tensors are on one HIP device; work goes to torch's current stream of that device, where the
outputs and workspaces are allocated too.  Tensors that do not fit raise ``ValueError``, sizes and
options out of the kernels' range ``gsn.GsnError``.
"""
from __future__ import annotations

import functools

import torch
from torch.autograd import forward_ad

from . import gsn


# (the checks of a call cost a single token as much as its kernel: they are kept short)
def _same_device(x, *others):
    d = x.get_device()
    for t in others:
        if t is not None and t.get_device() != d:
            raise ValueError(f"a tensor of {tuple(t.shape)} is on {t.device}, not on {x.device}")


def _no_tangent(*tensors):
    """Refuses tensors with a forward-mode tangent, which the kernels would drop."""
    if getattr(forward_ad, "_current_level", 0) < 0:  # outside of any dual_level: the usual case
        return
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"a tensor of {tuple(t.shape)} carries a forward-mode tangent; "
                             "there is no forward-mode derivative")


class _Once(torch.autograd.Function):
    """The first ``count`` tensors, gradients computed from the others; raises where they are
    differentiated."""

    @staticmethod
    def forward(ctx, what, count, *tensors):
        ctx.what = what
        return tensors[:count]

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"the gradients of {ctx.what} cannot be differentiated a second time")


def _once(what, grads, *of):
    """The gradients that a backward method returns, made of the tensors ``of``.  In a backward
    pass that is itself recorded (create_graph=True) they would else count as constants."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in of):
        return _Once.apply(what, len(grads), *grads, *of)
    return grads


def _rows(x: torch.Tensor, what: str) -> torch.Tensor:
    if x.dim() != 2:
        raise ValueError(f"{what} must be 2-dimensional, got {tuple(x.shape)}")
    return x


def _bytes(n: int, x: torch.Tensor) -> torch.Tensor:
    # torch's allocator aligns to 512 bytes
    return x.new_empty(n, dtype=torch.uint8)


# ----------------------------------------------------------------------- layer norm ----

def layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """(y, stats): the norm of every row of x (rows, dim) and what its backward pass takes."""
    _rows(x, "x")
    _same_device(x, weight, bias)
    y = torch.empty_like(x)
    stats = x.new_empty(2, x.shape[0], dtype=torch.float32)
    gsn.gsn_layer_norm(x, weight, bias, eps, y, stats)
    return y, stats


def layer_norm_backward(dy, x, weight, bias, stats, need=(True, True, True)):
    """(dx, dweight, dbias) from dy; None for what is not needed or has no parameter."""
    _rows(x, "x")
    _same_device(x, dy, weight, bias, stats)
    rows, dim = x.shape
    dx = torch.empty_like(x) if need[0] else None
    dweight = torch.empty_like(weight) if need[1] and weight is not None else None
    dbias = torch.empty_like(bias) if need[2] and bias is not None else None
    ws = None
    if dweight is not None or dbias is not None:
        ws = _bytes(gsn.gsn_layer_norm_workspace_bytes(rows, dim), x)
    gsn.gsn_layer_norm_backward(dy, x, weight, stats, dx, dweight, dbias, ws)
    return dx, dweight, dbias


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, stats = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, bias, stats)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, stats = ctx.saved_tensors
        if dy.stride(-1) != 1 or (dy.shape[0] > 1 and dy.stride(0) < dy.shape[1]):
            dy = dy.contiguous()  # (an expanded gradient, as that of a sum)
        grads = layer_norm_backward(dy, x, weight, bias, stats, ctx.needs_input_grad)
        return (*_once("layer_norm", grads, dy, x, weight), None)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension of x (rows, dim).  weight and bias: (dim,), float32 or
    of x's type, or None.  Rows may be those of a wider tensor (any row stride)."""
    _no_tangent(x, weight, bias)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad
                                       for t in (x, weight, bias)):
        return _LayerNorm.apply(x, weight, bias, eps)
    _rows(x, "x")
    _same_device(x, weight, bias)
    y = torch.empty_like(x)
    gsn.gsn_layer_norm(x, weight, bias, eps, y)
    return y


# -------------------------------------------------------------------------- routing ----

_route_params = functools.lru_cache(maxsize=256)(gsn.make_route)  # (never written to)


def _route(logits, params, balance, valid):
    _same_device(logits, balance, valid)
    tokens = logits.shape[0]
    ids = logits.new_empty(tokens, params.top, dtype=torch.int32)
    weights = logits.new_empty(tokens, params.top, dtype=torch.float32)
    gsn.gsn_route(params, logits, balance, valid, ids, weights)
    return ids, weights


def _route_backward(dweights, logits, ids, params):
    _same_device(logits, dweights, ids)
    dlogits = torch.empty_like(logits)
    gsn.gsn_route_backward(params, dweights, logits, ids, dlogits)
    return dlogits


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, params, balance, valid):
        ids, weights = _route(logits, params, balance, valid)
        ctx.params = params
        ctx.save_for_backward(logits, ids)
        ctx.mark_non_differentiable(ids)
        return ids, weights

    @staticmethod
    def backward(ctx, _, dweights):
        logits, ids = ctx.saved_tensors
        dlogits = _route_backward(dweights.contiguous(), logits, ids, ctx.params)
        return *_once("route", (dlogits,), dweights, logits), None, None, None


def route(logits, top, *, score="softmax", balance=None, groups=1, top_groups=1, best=1,
          renormalise=True, scale=1.0, valid=None):
    """(ids, weights), each (tokens, top): the best experts of every token, by descending order,
    and their weights; see gsn_route in include/gsn.h for the order, masks and ties.  The weights
    are differentiable with respect to the logits."""
    _rows(logits, "logits")
    _no_tangent(logits, balance)
    params = _route_params(logits.shape[1], top, score, groups, top_groups, best, renormalise,
                           scale)
    if torch.is_grad_enabled() and logits.requires_grad:
        return _Route.apply(logits, params, balance, valid)
    return _route(logits, params, balance, valid)


def route_backward(dweights, logits, ids, *, score="softmax", groups=1, top_groups=1, best=1,
                   renormalise=True, scale=1.0):
    """dlogits of ``route`` with the same options (those of the choice alone do not matter)."""
    _rows(logits, "logits")
    params = _route_params(logits.shape[1], ids.shape[1], score, groups, top_groups, best,
                           renormalise, scale)
    return _route_backward(dweights, logits, ids, params)


def route_counts(ids, experts):
    """Pairs of each expert, int32 (experts,)."""
    counts = torch.empty(experts, dtype=torch.int32, device=ids.device)
    gsn.gsn_route_counts(ids, counts)
    return counts


def route_balance(counts, balance, rate=1e-3):
    """Moves balance in place by rate towards the experts with fewer pairs than the mean."""
    _same_device(counts, balance)
    gsn.gsn_route_balance(counts, rate, balance)
    return balance


# ------------------------------------------------------------------- experts' products ----

def _experts_forward(x, ids, weights, w1, w2, save):
    _rows(x, "x")
    _same_device(x, ids, weights, w1, w2)
    p = gsn.make_experts(x, ids, w1, w2)
    size = gsn.gsn_experts_workspace_bytes(p, False)
    if size == 0:
        raise gsn.GsnError(gsn.GSN_E_INVAL, "gsn_experts_workspace_bytes")
    out = torch.empty_like(x, memory_format=torch.contiguous_format)
    saved = _bytes(gsn.gsn_experts_saved_bytes(p), x) if save else None
    gsn.gsn_experts(p, x, ids, weights, w1, w2, out, saved, _bytes(size, x))
    return out, saved


def experts_forward(x, ids, weights, w1, w2):
    """(out, saved): the experts' products and what their backward pass takes."""
    return _experts_forward(x, ids, weights, w1, w2, True)


def experts_backward(dout, x, ids, weights, w1, w2, saved, need=(True, True, True, True)):
    """(dx, dweights, dw1, dw2) from dout; None for what is not needed."""
    _rows(x, "x")
    _same_device(x, dout, ids, weights, w1, w2, saved)
    p = gsn.make_experts(x, ids, w1, w2)
    size = gsn.gsn_experts_workspace_bytes(p, True)
    if size == 0:
        raise gsn.GsnError(gsn.GSN_E_INVAL, "gsn_experts_workspace_bytes")
    dx, dweights, dw1, dw2 = (
        torch.empty_like(t, memory_format=torch.contiguous_format) if n else None
        for t, n in zip((x, weights, w1, w2), need))
    gsn.gsn_experts_backward(p, dout, x, weights, w1, w2, saved, dx, dweights, dw1, dw2,
                             _bytes(size, x))
    return dx, dweights, dw1, dw2


class _Experts(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, ids, weights, w1, w2):
        out, saved = experts_forward(x, ids, weights, w1, w2)
        ctx.save_for_backward(x, ids, weights, w1, w2, saved)
        return out

    @staticmethod
    def backward(ctx, dout):
        x, ids, weights, w1, w2, saved = ctx.saved_tensors
        need = ctx.needs_input_grad
        grads = experts_backward(dout.contiguous(), x, ids, weights, w1, w2, saved,
                                 (need[0], *need[2:5]))
        dx, *rest = _once("experts", grads, dout, x, weights, w1, w2)
        return dx, None, *rest


def experts(x, ids, weights, w1, w2):
    """out[t] = sum_k weights[t, k] * w2[e] (silu(gate) * up), (gate, up) = w1[e] x[t] and
    e = ids[t, k].  x (tokens, dim), ids int32 and weights float32 (tokens, top), w1 (experts,
    2 * hidden, dim) with the gate's rows first, w2 (experts, dim, hidden).  A pair whose id is
    not an expert's adds nothing.  silu(gate) * up, and the gradients of gate and up, are rounded
    to x's type between the products: in float16 they have its range (include/gsn.h), and a loss
    is scaled as usual there."""
    _no_tangent(x, weights, w1, w2)
    if torch.is_grad_enabled() and any(t.requires_grad for t in (x, weights, w1, w2)):
        return _Experts.apply(x, ids, weights, w1, w2)
    return _experts_forward(x, ids, weights, w1, w2, False)[0]
