"""Training and serving models over the units of a network, on torch tensors, through the C calls of
``include/gsn.h``.

A network of units is a vocabulary: what a signal is to it is its winner.  A model that answers with
a unit has its units as classes: ``cross_entropy`` is that model's loss, without keeping the logits
of all units.  ``orthogonal_step`` updates its matrices and those of the local experts of
``mixture`` by the orthogonalised momentum of their gradients, ``linear_8bit`` serves a layer in 8
bits.  ``cross_entropy`` takes part in autograd, once: derivatives of its gradients raise
``RuntimeError``; ``cross_entropy_forward`` and ``cross_entropy_backward`` are its two halves for
programs that keep their own order.  The other calls have no derivatives and refuse tensors that
want them, and all refuse tensors that carry a forward-mode tangent.

Tensors are on one HIP device; work goes to torch's current stream of that device, where the
outputs and workspaces are allocated too.  Tensors that do not fit raise ``ValueError``, sizes and
options out of the kernels' range ``gsn.GsnError``.  All calls can be recorded into a HIP graph; a
backward pass through autograd, as any of torch's, only while no eager graph of the same leaves
lives.
"""
from __future__ import annotations

import functools

import torch

from . import gsn
from .gsn import _int32
from .mixture import _bytes, _no_tangent, _once, _rows, _same_device

COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # five steps take singular values of 0.002 to 1 near 1


# (parameters and workspace sizes go by sizes and types alone: they are made once for each of them,
# and never written to)
def _sized(name: str, p, size: int):
    if size == 0:
        raise gsn.GsnError(gsn.GSN_E_INVAL, name)
    return p, size


@functools.lru_cache(maxsize=256)
def _entropy(code, dim, classes, tokens, backward):
    p = gsn.gsn_entropy_params(code, _int32(dim), _int32(classes), tokens)
    return _sized("gsn_cross_entropy", p, gsn.gsn_cross_entropy_workspace_bytes(p, backward))


@functools.lru_cache(maxsize=256)
def _orthogonal(code, rows, cols, batch, steps, coefficients, eps, update):
    p = gsn.gsn_orthogonal_params(code, _int32(rows), _int32(cols), _int32(steps), batch,
                                  *coefficients, eps)
    return _sized("gsn_orthogonalise", p, gsn.gsn_orthogonal_workspace_bytes(p, update))


@functools.lru_cache(maxsize=256)
def _linear(code, dim, out, tokens):
    p = gsn.gsn_linear_params(code, _int32(dim), _int32(out), tokens)
    return _sized("gsn_linear_quantised", p, gsn.gsn_linear_quantised_workspace_bytes(p))


def _no_gradient(what: str, *tensors):
    """Refuses tensors that want a gradient, which would not get one."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError(f"{what} has no derivative: call it under torch.no_grad(), or with "
                         "detached tensors")


def _written(*tensors):
    """Counts as a write to them for autograd, as an operation of torch's in place does: what was
    saved of them for a backward pass is no longer what it was."""
    for t in tensors:
        if not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _operands(x, w):
    """(type, columns of both, rows of w, rows of x) of the operands of x w^T."""
    if w.dim() != 2:
        raise ValueError(f"w must be 2-dimensional, got {tuple(w.shape)}")
    tokens, dim = x.shape
    return gsn._type(x, "x"), dim, w.shape[0], tokens


# -------------------------------------------------------------------- cross entropy ----

def _cross_entropy(x, w, targets, valid, save):
    _rows(x, "x")
    _same_device(x, w, targets, valid)
    p, size = _entropy(*_operands(x, w), False)
    loss = x.new_empty(x.shape[0], dtype=torch.float32)
    stats = x.new_empty(2, x.shape[0], dtype=torch.float32) if save else None
    gsn.gsn_cross_entropy(p, x, w, targets, valid, loss, stats, _bytes(size, x))
    return loss, stats


def cross_entropy_forward(x, w, targets, valid=None):
    """(loss, stats): the loss of every token and what the backward pass takes."""
    _no_tangent(x, w)
    return _cross_entropy(x, w, targets, valid, True)


def cross_entropy_backward(dloss, x, w, targets, valid, stats, need=(True, True)):
    """(dx, dw) from dloss (tokens,) float32; None for what is not needed."""
    _no_tangent(dloss, x, w, stats)
    _rows(x, "x")
    _same_device(x, dloss, w, targets, valid, stats)
    p, size = _entropy(*_operands(x, w), True)
    dx, dw = (torch.empty_like(t, memory_format=torch.contiguous_format) if n else None
              for t, n in zip((x, w), need))
    gsn.gsn_cross_entropy_backward(p, dloss, x, w, targets, valid, stats, dx, dw,
                                   _bytes(size, x))
    return dx, dw


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, targets, valid):
        loss, stats = cross_entropy_forward(x, w, targets, valid)
        ctx.save_for_backward(x, w, targets, valid, stats)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, w, targets, valid, stats = ctx.saved_tensors
        grads = cross_entropy_backward(dloss.contiguous(), x, w, targets, valid, stats,
                                       ctx.needs_input_grad[:2])
        return (*_once("cross_entropy", grads, dloss, x, w), None, None)


def cross_entropy(x, w, targets, valid=None):
    """loss[t] = log(sum_c exp(x[t] . w[c])) - x[t] . w[targets[t]], float32 (tokens,), over the
    valid classes c.  x (tokens, dim) and w (classes, dim), rows of wider tensors as they may be;
    targets int32 (tokens,); valid uint8 (classes,) or None.  A token whose target is out of range
    or not valid has the loss 0 and no gradient, whatever its x; a class that is not valid is in no
    sum, whatever its row of w.  The logits are never kept as a whole; the backward pass makes
    them again."""
    _no_tangent(x, w)
    if torch.is_grad_enabled() and (x.requires_grad or w.requires_grad):
        return _CrossEntropy.apply(x, w, targets, valid)
    return _cross_entropy(x, w, targets, valid, False)[0]


# -------------------------------------------------------------- orthogonalised updates ----

def _matrices(x):
    """(type, rows, columns, number) of the matrices of x."""
    if x.dim() < 2:
        raise ValueError(f"a matrix or a batch of them is needed, got {tuple(x.shape)}")
    rows, cols = x.shape[-2:]
    if rows == 0 or cols == 0:
        raise ValueError(f"matrices without elements: {tuple(x.shape)}")
    return gsn._type(x, "x"), rows, cols, x.numel() // (rows * cols)


def orthogonalise(x, *, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The orthogonalised matrices of x (..., rows, cols): their singular vectors with singular
    values near 1 (0.7 to 1.2 with the usual coefficients and steps, where a value is above some
    0.002 of the matrix's norm).  See gsn_orthogonalise in include/gsn.h for the products."""
    _no_tangent(x)
    _no_gradient("orthogonalise", x)
    p, size = _orthogonal(*_matrices(x), steps, tuple(map(float, coefficients)),
                          float(eps), False)
    x = x.contiguous()
    out = torch.empty_like(x)
    gsn.gsn_orthogonalise(p, x, out, _bytes(size, x))
    return out


def orthogonal_step(weights, gradient, momentum, rate, *, beta=0.95, nesterov=True, decay=0.0,
                    scale=None, steps=5, coefficients=COEFFICIENTS, eps=1e-7, out=None):
    """(weights, momentum) after one update of matrices (..., rows, cols):

        momentum = beta * momentum + gradient
        weights = (1 - rate * decay) * weights
                  - rate * scale * orthogonalise(gradient + beta * momentum)

    (of the momentum alone without nesterov).  scale: sqrt(max(1, rows / cols)) if None, so that
    the update moves outputs as far whatever the shape.  momentum is float32, gradient of the type
    of weights, all contiguous.  out: the two tensors that take the results, (weights, momentum) for
    an update in place, which autograd sees as one; new ones if None."""
    given = () if out is None else tuple(out)
    _no_tangent(weights, gradient, momentum, *given)
    _no_gradient("orthogonal_step", weights, gradient, momentum, *given)
    p, size = _orthogonal(*_matrices(weights), steps, tuple(map(float, coefficients)), float(eps),
                          True)
    new_weights, new_momentum = given if out is not None else (
        torch.empty_like(weights, memory_format=torch.contiguous_format),
        torch.empty_like(momentum, memory_format=torch.contiguous_format))
    _same_device(weights, gradient, momentum, new_weights, new_momentum)
    if scale is None:
        scale = max(1.0, p.rows / p.cols) ** 0.5
    gsn.gsn_orthogonal_step(p, weights, gradient, momentum, rate * scale, beta, rate * decay,
                            nesterov, new_weights, new_momentum, _bytes(size, weights))
    _written(*given)
    return new_weights, new_momentum


# -------------------------------------------------------------------- products in 8 bits ----

def quantise(x):
    """(q, scales) of the rows of x (rows, dim): q int8 with x near q * scales[:, None], scales
    float32 (rows,), the largest |x| of a row over 127.  The rows of q start at multiples of 16
    bytes, as linear_8bit reads them fastest."""
    _rows(x, "x")
    _no_tangent(x)
    _no_gradient("quantise", x)
    rows, dim = x.shape
    q = x.new_empty(rows, (dim + 15) // 16 * 16, dtype=torch.int8)[:, :dim]
    scales = x.new_empty(rows, dtype=torch.float32)
    gsn.gsn_quantise(x, q, scales)
    return q, scales


def linear_8bit(x, w, scales):
    """y = (q w^T) * s[:, None] * scales, (q, s) = quantise(x): x (tokens, dim) through a layer
    whose weights w int8 (out, dim) and scales float32 (out,) quantise() made.  Sums are exact;
    y is of x's type."""
    _rows(x, "x")
    _no_tangent(x)
    _no_gradient("linear_8bit", x, scales)
    _same_device(x, w, scales)
    p, size = _linear(*_operands(x, w))
    y = x.new_empty(x.shape[0], w.shape[0])
    gsn.gsn_linear_quantised(p, x, w, scales, y, _bytes(size, x))
    return y
