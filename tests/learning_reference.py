"""Plain 64-bit definitions of the operators that train and serve a model over a network's units
(torch on the CPU), and the errors that their arithmetic may have, for the tests to compare with."""
import numpy as np
import torch

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half of the smallest step of the type
HALF_STEP = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U = 2.0 ** -24
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


# -------------------------------------------------------------------- cross entropy ----

def cross_entropy(x, w, targets, valid=None, dloss=None):
    """A dict with loss, dx, dw and, for each, how far a result of the kernels may be off: *_tol.

    A logit is a sum of dim products in binary32, off by at most dim U sum |x w| (U = 2^-24): E at
    most for a token.  Binary32 operands may be kept in two float16 values: each element to 2^-23 of
    itself (and 2^-40 of its row's largest), the product of the two last ones, 2^-22 at most, left
    out: 8 U more.  exp(l - largest) is off by that twice, by (|l - largest| + 3) 2 U of the
    exponential (its argument and itself), and the sum of the exponentials by one U for each of the
    additions that a term goes through, 64 + classes / 64 at most.  The gradients of the logits are
    rounded to the operands' type, those of float16 as multiples of 2^-15 of the largest dloss; in
    two values to 2^-23, and to 2^-36 of the largest that one could be beside w's, or x's, largest.
    Their products with w and x are sums of binary32, the results are rounded once."""
    dtype = x.dtype
    classes, dim = w.shape
    there = torch.ones(classes, dtype=torch.bool) if valid is None else valid != 0
    t = targets.long()
    live = (t >= 0) & (t < classes)
    at = t.clamp(0, classes - 1)
    live &= there[at]
    x = torch.where(live[:, None], x.double(), 0.0)
    w = torch.where(there[:, None], w.double(), 0.0)
    l = (x @ w.t()).masked_fill(~there, -torch.inf)
    size = (x.abs() @ w.abs().t()).masked_fill(~there, 0.0)
    two = dtype == torch.float32
    err = (dim + 8 * two) * U * size.max(1, keepdim=True)[0] \
        + two * dim * 2.0 ** -39 * x.abs().max() * w.abs().max()
    top = l.max(1, keepdim=True)[0]
    top = torch.where(top == -torch.inf, 0.0, top)
    e = torch.exp(l - top)
    total = e.sum(1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    log_total = torch.log(total.clamp(min=1e-300))
    chosen = l.gather(1, at[:, None])
    rel_sum = 2 * err + (64 + classes / 64) * U \
        + (p * torch.where(p > 0, (l - top).abs() + 3, 0.0)).sum(1, keepdim=True) * 2 * U
    loss = torch.where(live, (log_total + top - chosen)[:, 0], 0.0)
    parts = log_total.abs() + (chosen - top).abs().nan_to_num(0.0, 0.0, 0.0)
    out = {"loss": loss, "loss_tol": torch.where(
        live, (3 * err + rel_sum + 8 * U * (parts + 1))[:, 0], 0.0)}
    if dloss is None:
        return out
    g = torch.where(live, dloss.double(), 0.0)[:, None]
    d = p.clone()
    d.scatter_add_(1, at[:, None], torch.full_like(chosen, -1.0))
    d = d * g
    rel_p = rel_sum + 2 * err + (torch.where(p > 0, (l - top).abs(), 0.0) + 3) * 2 * U
    ulp = 2.0 ** -23 if two else HALF_ULP[dtype]
    step = HALF_STEP[dtype]
    if dtype == torch.float16:
        step = step * 2.0 ** -15 * g.abs().max()
    d_tol = (p * rel_p + 4 * U) * g.abs() + ulp * d.abs() + step
    d_tol = torch.where(live[:, None] & there, d_tol, 0.0)
    for name, a, b in (("dx", d, w), ("dw", d.t(), x)):
        tol = d_tol if name == "dx" else d_tol.t()
        v = a @ b
        out[name] = v
        out[name + "_tol"] = (tol + (a.shape[1] + 12) * U * (a.abs() + tol)) @ b.abs() * (1 + ulp) \
            + ulp * v.abs() + HALF_STEP[dtype]
        if two:
            out[name + "_tol"] += a.shape[1] * 2.0 ** -34 * b.abs().max() * (
                g.abs() if name == "dx" else g.abs().max())
    return out


# -------------------------------------------------------------- orthogonalised matrices ----

def orthogonalise(x, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The definition, of one matrix or a batch, in float64."""
    a, b, c = coefficients
    x = x.double()
    if x.numel() == 0:
        return x
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    norm = x.square().sum((-2, -1), keepdim=True).sqrt() + eps
    x = torch.where(norm > 0, x / norm, 0.0)
    for _ in range(steps):
        k = x @ x.mT
        x = a * x + (b * k + c * (k @ k)) @ x
    return x.mT if tall else x


def orthogonal_error(x, values, steps=5, coefficients=COEFFICIENTS):
    """How far (2-norm of all entries) the kernels' result may be from the definition's of one
    matrix x, before its own rounding.

    The exact iterates have the singular values s of x / norm, taken through f(s) = s (a + b s^2 +
    c s^4).  A matrix that is kept is off by `keep` of its norm: 2^-11 with one float16 value, 2^-22
    with two, of which the products leave the last, lo lo, out: 2^-22 more.  A product of k terms a
    sum is off by sum_k = 4 sqrt(3 k) U of the product of the norms of its factors: rounding errors
    of a sum as independent ones, four of their standard deviations (U = 2^-24).  What a step adds
    is passed on by the rest of the steps: a function of the singular values takes a small change
    of its matrix times the largest of (f(s) - f(t)) / (s - t) and (f(s) + f(t)) / (s + t) over
    their pairs."""
    a, b, c = coefficients
    x = x.double()
    s = torch.linalg.svdvals(x)
    s = (s / s.norm()).numpy()
    short, long = min(x.shape), max(x.shape)
    keep = 2.0 ** -11 if values == 1 else 2 * 2.0 ** -22

    def f(v):
        return v * (a + (b + c * v * v) * v * v)

    def passes(v0, v):
        """The largest divided difference of v0 -> v over pairs of both signs."""
        p, q = np.concatenate([v0, -v0]), np.concatenate([v, -v])
        dp = p[:, None] - p[None, :]
        dq = q[:, None] - q[None, :]
        h = 1e-6 * (np.abs(p).max() + 1)
        far = np.abs(dp) > h
        most = np.abs(np.where(far, dq / np.where(far, dp, 1.0), 0.0)).max()
        return most

    orbit = [s]
    for _ in range(steps):
        orbit.append(f(orbit[-1]))
    slope = []  # of one step, and of the steps after it, where they are near each other
    for v in orbit[:-1]:
        slope.append(np.abs(a + 3 * b * v ** 2 + 5 * c * v ** 4))
    error = 0.0
    for i in range(steps):
        v = np.abs(orbit[i])
        norm, most = np.sqrt((v ** 2).sum()), v.max()
        gram, gram_most = np.sqrt((v ** 4).sum()), most ** 2
        poly = a + b * v ** 2 + c * v ** 4
        poly_norm, poly_most = np.sqrt((poly ** 2).sum()), np.abs(poly).max()
        # x kept (the first too: times 2^11 / norm it is rounded), A, B and the new x
        e_x = keep * norm
        e_a = 2 * most * e_x + 4 * np.sqrt(3 * long) * U * norm * norm + keep * gram
        e_b = abs(b) * e_a + abs(c) * (2 * gram_most * e_a +
                                       4 * np.sqrt(3 * short) * U * gram * gram) \
            + keep * poly_norm
        e_next = poly_most * e_x + most * e_b + 4 * np.sqrt(3 * short) * U * poly_norm * norm
        near = np.ones_like(v)
        for k in range(i + 1, steps):
            near = near * slope[k]
        left = max(1.0 if i + 1 == steps else passes(orbit[i + 1], orbit[-1]), near.max())
        error += left * e_next
    return 1.05 * error


# -------------------------------------------------------------------- products in 8 bits ----

def quantise(x):
    """(q int64, scales float32, exact) of the rows of x."""
    v = x.float().numpy()
    top = np.abs(v).max(1) if v.shape[1] else np.zeros(len(v), np.float32)
    bad = ~np.isfinite(top)
    with np.errstate(invalid="ignore"):
        s = np.maximum(top / np.float32(127), np.float32(2.0 ** -126)).astype(np.float32)
        q = np.rint(v.astype(np.float64) / s.astype(np.float64)[:, None])
    q = np.where(bad[:, None], 0, np.clip(np.nan_to_num(q), -127, 127))
    return torch.from_numpy(q.astype(np.int64)), torch.from_numpy(
        np.where(bad, np.float32(np.nan), s).astype(np.float32))


def linear_8bit(x, w, scales):
    """(y float64, tolerance): three roundings of 2^-24 (the integer, two products), then one to the
    type."""
    q, s = quantise(x)
    y = (q @ w.long().t()).double() * s.double()[:, None] * scales.double()
    return y, y.abs() * (HALF_ULP[x.dtype] + 4 * U) + HALF_STEP[x.dtype]
