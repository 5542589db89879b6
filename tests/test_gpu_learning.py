"""The cross entropy, the orthogonalised updates and the products in 8 bits on the GPU against their
64-bit definitions: types, odd sizes, strides, tokens without a target, classes that are not there,
gradients against the formulas and against differences, other streams, recorded graphs."""
import numpy as np
import pytest
import torch

import learning_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def learn():
    from paper_1503_08294_amd import learning
    return learning


def randn(*shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def randint(lo, hi, *shape, seed):
    return torch.randint(lo, hi, shape, generator=torch.Generator().manual_seed(seed))


def close(got, want, tol, what):
    """|got - want| <= tol elementwise, no NaN."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - tol).max().item() if got.numel() else 0.0
    assert over <= 0, f"{what}: {over} beyond the tolerance"


# -------------------------------------------------------------------- cross entropy ----

def entropy_inputs(tokens, dim, classes, dtype, seed, shut=0.0, lost=0.0):
    w = randn(classes, dim, seed=seed, dtype=dtype, scale=1.5 * dim ** -0.5)
    t = randint(0, classes, tokens, seed=seed + 1).int()
    known = 4 * torch.rand(tokens, 1, generator=torch.Generator().manual_seed(seed + 2))
    x = (randn(tokens, dim, seed=seed + 3) + known * w[t.long()].float()).to(dtype)
    valid = None
    if shut:
        valid = (torch.rand(classes, generator=torch.Generator().manual_seed(seed + 4))
                 >= shut).to(torch.uint8)
    if lost:
        t[torch.rand(tokens, generator=torch.Generator().manual_seed(seed + 5)) < lost] = -1
    dloss = randn(tokens, seed=seed + 6) / tokens
    return x, w, t, valid, dloss


def check_entropy(learn, x, w, t, valid, dloss, what, view=lambda v: v.cuda()):
    want = ref.cross_entropy(x, w, t, valid, dloss)
    xd, wd = view(x), view(w)
    td, vd = t.cuda(), None if valid is None else valid.cuda()
    loss, stats = learn.cross_entropy_forward(xd, wd, td, vd)
    close(loss, want["loss"], want["loss_tol"], f"{what} loss")
    alone = learn.cross_entropy(xd, wd, td, vd)
    close(alone, want["loss"], want["loss_tol"], f"{what} loss alone")
    dx, dw = learn.cross_entropy_backward(dloss.cuda(), xd, wd, td, vd, stats)
    assert dx.dtype == x.dtype and dw.dtype == w.dtype and loss.dtype == F32
    close(dx, want["dx"], want["dx_tol"], f"{what} dx")
    close(dw, want["dw"], want["dw_tol"], f"{what} dw")
    return dx, dw


# (from 192 tokens on binary32 operands are kept in two float16 values)
SIZES = [(191, 40, 90), (192, 40, 90), (193, 1, 3), (1, 1, 1), (1, 64, 100), (2, 8, 7),
         (3, 5, 129), (17, 33, 65), (64, 64, 64),
         (65, 128, 257), (130, 72, 513), (129, 501, 333), (257, 256, 1000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,dim,classes", SIZES)
def test_entropy_forward_and_backward(learn, dtype, tokens, dim, classes):
    check_entropy(learn, *entropy_inputs(tokens, dim, classes, dtype, 1), f"{dtype}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,dim,classes", [(5, 16, 40), (70, 65, 200), (131, 64, 300)])
def test_entropy_masks(learn, dtype, tokens, dim, classes):
    x, w, t, valid, dloss = entropy_inputs(tokens, dim, classes, dtype, 2, shut=0.3, lost=0.2)
    t[0] = classes + 3  # out of range at the other end
    valid[t[1]] = 0     # a class that is not there as a target
    lost = (t < 0) | (t >= classes)
    lost |= valid[t.clamp(0, classes - 1).long()] == 0
    x[lost] = torch.nan
    w[valid == 0] = torch.inf
    dloss[lost] = torch.nan
    dx, dw = check_entropy(learn, x, w, t, valid, dloss, f"{dtype}")
    assert (dx[lost.cuda()] == 0).all() and (dw[valid.cuda() == 0] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_entropy_of_nothing(learn, dtype):
    """Every class shut, no token with a target, no token at all."""
    x, w, t, _, dloss = entropy_inputs(20, 40, 30, dtype, 3)
    none = torch.zeros(30, dtype=torch.uint8)
    check_entropy(learn, x, w, t, none, dloss, "no class")
    check_entropy(learn, x, w, torch.full_like(t, -5), None, dloss, "no target")
    loss, stats = learn.cross_entropy_forward(x[:0].cuda(), w.cuda(), t[:0].cuda())
    assert loss.shape == (0,)
    dx, dw = learn.cross_entropy_backward(dloss[:0].cuda(), x[:0].cuda(), w.cuda(), t[:0].cuda(),
                                          None, stats)
    assert dx.shape == (0, 40) and (dw == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,pad", [(64, 1), (64, 8), (33, 7), (40, 24)])
def test_entropy_strides(learn, dtype, dim, pad):
    """Rows cut out of wider buffers, whose other columns are not numbers."""
    def wide(v):
        b = torch.full((v.shape[0], v.shape[1] + 2 * pad), torch.nan, dtype=v.dtype)
        b[:, pad:-pad] = v
        return b.cuda()[:, pad:-pad]

    check_entropy(learn, *entropy_inputs(70, dim, 150, dtype, 4), f"{dtype}", wide)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 200])
def test_entropy_of_an_impossible_target(learn, dtype, tokens):
    """A target whose logit is -inf has an infinite loss; the other tokens keep theirs."""
    x, w, t, _, _ = entropy_inputs(tokens, 24, 50, dtype, 14)
    x[1] = 0
    x[1, 3] = torch.inf
    w[:, 3] = w[:, 3].abs() + 0.1
    w[t[1].long(), 3] = -1
    w[:, 3] *= -1  # every logit of token 1 is -inf but its target's, which is inf: NaN
    t[2] = t[1]
    loss = learn.cross_entropy(x.cuda(), w.cuda(), t.cuda()).cpu()
    assert torch.isnan(loss[1])
    w[:, 3] *= -1  # every logit is inf but the target's: NaN too, as inf - inf is
    loss = learn.cross_entropy(x.cuda(), w.cuda(), t.cuda()).cpu()
    assert not torch.isfinite(loss[1])
    keep = torch.arange(tokens) != 1
    want = ref.cross_entropy(x[keep], w, t[keep])
    close(loss[keep], want["loss"], want["loss_tol"], "the others")


@pytest.mark.parametrize("dtype", TYPES)
def test_entropy_large_and_small_logits(learn, dtype):
    """Logits of some hundreds (exp would overflow), a token that is sure, and a dloss far below the
    others'."""
    x, w, t, _, dloss = entropy_inputs(40, 64, 90, dtype, 5)
    x[:10] *= 60
    x[10] = (50 * w[t[10].long()].float()).to(dtype)
    dloss[11] *= 2.0 ** -18
    dloss[12] = 0
    check_entropy(learn, x, w, t, None, dloss, f"{dtype}")


@pytest.mark.parametrize("dtype,tokens,dim,classes", [
    (BF16, 300, 128, 33_000), (F16, 2_100, 64, 9_000), (F32, 1_100, 72, 5_000),
    (BF16, 5_000, 264, 130), (F32, 40, 16, 40_000), (F32, 5_000, 264, 130),
    (F32, 300, 1_100, 900), (BF16, 300, 1_100, 2_000), (F16, 700, 520, 2_100),
    (BF16, 40, 33, 500), (F16, 61, 1_000, 700), (F32, 100, 48, 300), (F32, 70, 600, 1_000),
    (F32, 33, 130, 200), (BF16, 1_500, 300, 1_700), (F16, 40, 64, 50_001)])
def test_entropy_many_classes_or_tokens(learn, dtype, tokens, dim, classes):
    """Tiles of every size, groups of waves that share k, sums split up along the classes and along
    the tokens, few tokens of rows that begin anywhere."""
    check_entropy(learn, *entropy_inputs(tokens, dim, classes, dtype, 6, shut=0.02, lost=0.02),
                  f"{dtype}")


def test_entropy_rows_of_very_different_size(learn):
    """Binary32 in two values: tokens and classes 2^-30 to 2^30 times the others' size, zeros."""
    x, w, t, _, dloss = entropy_inputs(260, 48, 200, F32, 13)
    t[t < 10] += 20
    x[3] *= 2.0 ** -30
    x[4] = 0
    x[5] *= 2.0 ** -100
    w[2] *= 2.0 ** -40
    w[3] = 0
    w[4] *= 2.0 ** -120
    x[6] *= 2.0 ** 9
    dloss[7] *= 2.0 ** -40
    dx, dw = check_entropy(learn, x, w, t, None, dloss, "sizes")
    want = ref.cross_entropy(x, w, t, None, dloss)["dx"][3]
    # (a token's gradient does not depend on how small it is itself)
    assert (dx[3].double().cpu() - want).norm() <= 1e-5 * want.norm()
    z, v = torch.zeros_like(x), torch.zeros_like(w)
    check_entropy(learn, z, w, t, None, dloss, "tokens of zeros")
    check_entropy(learn, x, v, t, None, dloss, "classes of zeros")
    check_entropy(learn, x * 2.0 ** 100, w * 2.0 ** -100, t, None, dloss, "far from 1")


def test_entropy_in_pieces(learn):
    """So many tokens that a pass takes several pieces of the classes: the losses and gradients are
    those of the tokens a part at a time."""
    tokens, dim, classes = 600_000, 16, 1_500
    g = torch.Generator(device="cuda").manual_seed(7)
    w = (torch.randn(classes, dim, generator=g, device="cuda") * 0.5).to(BF16)
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(BF16)
    t = torch.randint(-1, classes, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.rand(tokens, generator=g, device="cuda")
    loss, stats = learn.cross_entropy_forward(x, w, t)
    dx, dw = learn.cross_entropy_backward(dloss, x, w, t, None, stats)
    some = torch.arange(0, tokens, 9_973)
    want = ref.cross_entropy(x[some].cpu(), w.cpu(), t[some].cpu(), None, dloss[some].cpu())
    close(loss[some], want["loss"], want["loss_tol"], "loss")
    close(dx[some], want["dx"], want["dx_tol"], "dx")
    total = torch.zeros(classes, dim, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for i in range(0, tokens, 100_000):
        s = slice(i, i + 100_000)
        live = (t[s] >= 0)[:, None]
        d = torch.softmax(x[s].double() @ w.double().t(), 1)
        d.scatter_add_(1, t[s].long().clamp(min=0)[:, None],
                       torch.full((d.shape[0], 1), -1.0, device="cuda", dtype=torch.float64))
        d = torch.where(live, d * dloss[s].double()[:, None], 0.0)
        total += d.t() @ x[s].double()
        size += d.abs().t() @ x[s].double().abs()
    # a rounding to bfloat16 and binary32 exponentials for each term, the sum in splits of some
    # thousand tokens, one rounding of the result
    tol = size * (2.0 ** -8 + 1e-4) + total.abs() * 2.0 ** -8
    close(dw, total.cpu(), tol.cpu(), "dw")


def test_entropy_gradient_against_differences(learn):
    x, w, t, valid, _ = entropy_inputs(6, 12, 30, F32, 8, shut=0.2, lost=0.2)
    cot = randn(6, seed=9)
    xd, wd = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    (learn.cross_entropy(xd, wd, t.cuda(), valid.cuda()) * cot.cuda()).sum().backward()

    def value(x, w):
        return (ref.cross_entropy(x, w, t, valid)["loss"] * cot.double()).sum()

    h = 1e-5
    for leaf, other, name in ((x, w, "x"), (w, x, "w")):
        v = randn(*leaf.shape, seed=10).double()
        up, down = leaf.double() + h * v, leaf.double() - h * v
        f = (lambda a: value(a, other)) if name == "x" else (lambda a: value(other, a))
        slope = (f(up) - f(down)) / (2 * h)
        got = ((xd if name == "x" else wd).grad.double().cpu() * v).sum()
        # the quotient's own error h^2 (third derivatives of some tens) and binary32
        assert abs(got - slope) <= 1e-5 * (1 + abs(slope)), name


def test_entropy_one_gradient_at_a_time(learn):
    x, w, t, valid, dloss = (v.cuda() for v in entropy_inputs(90, 40, 140, BF16, 11, shut=0.1))
    _, stats = learn.cross_entropy_forward(x, w, t, valid)
    dx, dw = learn.cross_entropy_backward(dloss, x, w, t, valid, stats)
    only, none = learn.cross_entropy_backward(dloss, x, w, t, valid, stats, (True, False))
    assert none is None and torch.equal(only, dx)
    none, only = learn.cross_entropy_backward(dloss, x, w, t, valid, stats, (False, True))
    assert none is None and torch.equal(only, dw)


def test_entropy_mean_through_autograd(learn):
    """An expanded gradient comes in, as of a sum; frozen weights get none."""
    x, w, t, _, _ = entropy_inputs(50, 32, 70, F32, 12, lost=0.1)
    n = int((t >= 0).sum())
    xd = x.cuda().requires_grad_()
    (learn.cross_entropy(xd, w.cuda(), t.cuda()).sum() / n).backward()
    want = ref.cross_entropy(x, w, t, None, torch.full((50,), 1 / n))
    close(xd.grad, want["dx"], want["dx_tol"], "dx")


# -------------------------------------------------------------- orthogonalised updates ----

def check_orthogonal(got, x, dtype, values, what, **kw):
    """Each matrix within its error's norm and the rounding to its type."""
    got = got.double().cpu().reshape(-1, *x.shape[-2:])
    want = ref.orthogonalise(x, **kw).reshape(got.shape)
    assert torch.isfinite(got).all(), what
    for i, m in enumerate(x.reshape(got.shape)):
        tol = ref.orthogonal_error(m, values, **{k: v for k, v in kw.items() if k != "eps"}) \
            + (want[i] * ref.HALF_ULP[dtype]).norm() + ref.HALF_STEP[dtype] * want[i].numel() ** .5
        off = (got[i] - want[i]).norm()
        assert off <= tol, f"{what} matrix {i}: {off} of {tol}"


MATRICES = [(1, 1, 1), (2, 1, 9), (3, 7, 1), (2, 8, 8), (1, 33, 65), (3, 64, 64), (2, 100, 67),
            (1, 129, 257), (2, 300, 130), (1, 200, 201)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols", MATRICES)
def test_orthogonalise(learn, dtype, batch, rows, cols):
    x = randn(batch, rows, cols, seed=20, dtype=dtype, scale=3.0)
    check_orthogonal(learn.orthogonalise(x.cuda()), x, dtype, 2, f"{dtype}")


@pytest.mark.parametrize("batch,rows,cols", [(1, 3, 5), (2, 64, 192), (1, 130, 77), (2, 520, 700),
                                             (20, 300, 260)])
@pytest.mark.parametrize("steps,coefficients", [(1, ref.COEFFICIENTS), (2, (2.0, -1.5, 0.5)),
                                                (10, (1.5, -0.5, 0.0))])
def test_orthogonalise_other_polynomials(learn, steps, coefficients, batch, rows, cols):
    """(After one step little is passed on: a bound that a product left out would break.)"""
    x = randn(batch, rows, cols, seed=21)
    got = learn.orthogonalise(x.cuda(), steps=steps, coefficients=coefficients)
    check_orthogonal(got, x, F32, 2, f"{steps}", steps=steps, coefficients=coefficients)


@pytest.mark.parametrize("rows,cols", [(300, 700), (700, 300), (64, 64), (1_000, 1_100)])
def test_orthogonalise_keeps_every_element(learn, rows, cols):
    """X <- X, three times: every element keeps its 22 bits, those beside a tie of float16 too."""
    x = randn(rows, cols, seed=28)
    got = learn.orthogonalise(x.cuda(), steps=3, coefficients=(1.0, 0.0, 0.0)).double().cpu()
    want = x.double() / (x.double().norm() + 1e-7)
    # 1 / norm and its product are rounded to binary32; what is kept three times is off by half a
    # step of the second value, 2^-23 of the number or 2^-36 of the norm; the sums are exact but for
    # a rounding each, as is the result
    tol = want.abs() * (3 * 2.0 ** -23 + 6 * ref.U) + 3 * 2.0 ** -36
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalise_extreme_sizes_and_zeros(learn, dtype):
    big, small = {F32: (1e30, 1e-30), BF16: (1e30, 1e-30), F16: (1e4, 1e-4)}[dtype]
    x = randn(4, 24, 40, seed=22)
    x = torch.stack([x[0] * big, x[1] * small, x[2], x[3] * 0]).to(dtype)
    got = learn.orthogonalise(x.cuda(), eps=0.0)
    check_orthogonal(got[:3], x[:3], dtype, 2, f"{dtype}", eps=0.0)
    assert (got[3] == 0).all()
    # a norm far below eps gives next to nothing
    got = learn.orthogonalise((x[1:2].float() * 1e-8).to(dtype).cuda(), eps=1.0)
    assert torch.isfinite(got).all() and got.abs().max() < 1e-3
    # one matrix that is not finite does not touch the others
    y = x.clone()
    y[1, 3, 5] = torch.inf
    got = learn.orthogonalise(y.cuda(), eps=0.0)
    assert torch.isnan(got[1].float()).all()
    check_orthogonal(got[[0, 2]], x[[0, 2]], dtype, 2, f"{dtype}", eps=0.0)


def test_orthogonalise_shapes(learn):
    x = randn(2, 3, 20, 30, seed=23)
    got = learn.orthogonalise(x.cuda())
    assert got.shape == x.shape
    check_orthogonal(got, x, F32, 2, "four dimensions")
    assert torch.equal(learn.orthogonalise(x[1, 2].cuda()), got[1, 2])
    # columns of another order: the transposed matrix's memory
    t = x[0].cuda().transpose(1, 2)
    check_orthogonal(learn.orthogonalise(t), x[0].transpose(1, 2), F32, 2, "transposed")
    assert learn.orthogonalise(x[:, :0].cuda()).shape == (2, 0, 20, 30)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols", [(1, 520, 1100), (5, 700, 300), (40, 136, 200),
                                             (14, 300, 260), (70, 300, 520), (70, 520, 300)])
def test_orthogonalise_larger(learn, dtype, batch, rows, cols):
    """Tiles of every size; after one step little is passed on, and the bound is tight."""
    x = randn(batch, rows, cols, seed=24, dtype=dtype)
    pick = sorted({0, batch // 2, batch - 1})
    for steps in (5, 1):
        got = learn.orthogonalise(x.cuda(), steps=steps)
        check_orthogonal(got[pick], x[pick], dtype, 2, f"{dtype}", steps=steps)


def test_orthogonal_step_of_a_large_batch(learn):
    """One float16 value a number, in the largest tiles."""
    w, g = (randn(70, 520, 300, seed=s, dtype=BF16) for s in (48, 49))
    m = randn(70, 520, 300, seed=50)
    got, got_m = learn.orthogonal_step(w.cuda(), g.cuda(), m.cuda(), 0.5, steps=2)
    for i in (0, 33, 69):
        want_m = 0.95 * m[i].double() + g[i].double()
        u = g[i].double() + 0.95 * want_m
        o = ref.orthogonalise(u, steps=2)
        want = w[i].double() - 0.5 * (520 / 300) ** 0.5 * o
        tol = 0.5 * (520 / 300) ** 0.5 * ref.orthogonal_error(u, 1, steps=2) * (1 + 2.0 ** -10) \
            + (want * 2.0 ** -8).norm() + 1e-5 * want.norm()
        assert (got[i].double().cpu() - want).norm() <= tol
        close(got_m[i], want_m, 3 * ref.U * (m[i].abs().double() + g[i].abs().double()), "momentum")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("rows,cols", [(48, 30), (30, 48), (1, 5), (131, 260)])
def test_orthogonal_step(learn, dtype, nesterov, rows, cols):
    w = randn(2, rows, cols, seed=25, dtype=dtype)
    g = randn(2, rows, cols, seed=26, dtype=dtype)
    m = randn(2, rows, cols, seed=27, scale=4.0)
    rate, beta, decay = 0.05, 0.9, 0.1
    got_w, got_m = learn.orthogonal_step(w.cuda(), g.cuda(), m.cuda(), rate, beta=beta,
                                         nesterov=nesterov, decay=decay)
    want_m = beta * m.double() + g.double()
    close(got_m, want_m, 3 * ref.U * (m.abs().double() + g.abs().double()), "momentum")
    u = g.double() + beta * want_m if nesterov else want_m
    scale = max(1.0, rows / cols) ** 0.5
    o = ref.orthogonalise(u)
    want = w.double() * (1 - rate * decay) - rate * scale * o
    for i in range(2):
        # (u is binary32: one or two more roundings of 2^-24, below a float16 value's)
        e = ref.orthogonal_error(u[i], 1 if dtype != F32 else 2) * (1 + 2.0 ** -10)
        tol = rate * scale * e + (want[i].abs() * ref.HALF_ULP[dtype]).norm() \
            + 4 * ref.U * (w[i].double().norm() + rate * scale * o[i].norm())
        off = (got_w[i].double().cpu() - want[i]).norm()
        assert off <= tol, f"{off} of {tol}"
    # in place
    wd, md = w.cuda(), m.cuda()
    out = learn.orthogonal_step(wd, g.cuda(), md, rate, beta=beta, nesterov=nesterov, decay=decay,
                                out=(wd, md))
    assert out[0] is wd and torch.equal(wd, got_w) and torch.equal(md, got_m)


# -------------------------------------------------------------------- products in 8 bits ----

def check_linear(learn, x, dtype, out, what, view=lambda v: v.cuda()):
    wq, ws = learn.quantise(randn(out, x.shape[1], seed=30, scale=x.shape[1] ** -0.5).cuda())
    want, tol = ref.linear_8bit(x, wq.cpu(), ws.cpu())
    for w in (wq, wq.contiguous()):
        close(learn.linear_8bit(view(x), w, ws), want, tol, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 15), (2, 16), (5, 257), (64, 1024), (9, 4099)])
def test_quantise(learn, dtype, rows, dim):
    x = randn(rows, dim, seed=31, dtype=dtype) * torch.logspace(-3, 3, rows)[:, None].to(dtype)
    q, s = learn.quantise(x.cuda())
    want_q, want_s = ref.quantise(x)
    assert torch.equal(s.cpu(), want_s)
    assert torch.equal(q.cpu().long(), want_q)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_borders_and_odd_rows(learn, dtype):
    """Values half way between two integers go to the even one; rows of zeros, of the smallest
    values, of the largest; rows that hold something that is not finite."""
    x = torch.zeros(9, 256)
    x[0] = (torch.arange(256) - 127.5).clamp(-127, 127)  # scale 1: ties
    x[1] = x[0] * 2.0 ** -8
    x[3, 7] = torch.finfo(dtype).max
    x[3, 9] = -torch.finfo(dtype).max / 3
    x[4] = torch.finfo(dtype).tiny * torch.linspace(-1, 1, 256)
    x[5, 0] = torch.finfo(dtype).smallest_normal
    x[6] = torch.linspace(-3, 5, 256)
    x[6, 3] = torch.nan
    x[7, 200] = -torch.inf
    x[8] = -0.0
    x = x.to(dtype)
    q, s = learn.quantise(x.cuda())
    want_q, want_s = ref.quantise(x)
    assert torch.equal(s.cpu().nan_to_num(-1), want_s.nan_to_num(-1))
    assert torch.equal(q.cpu().long(), want_q)
    y = learn.linear_8bit(x.cuda(), *learn.quantise(torch.eye(256)[:20].cuda()))
    assert torch.isnan(y[6:8].float()).all() and torch.isfinite(y[[0, 1, 2, 4, 5, 8]].float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,dim,out", [(1, 1, 1), (1, 64, 100), (1, 4096, 333), (2, 17, 33),
                                            (5, 16, 64), (16, 1000, 129), (17, 80, 70),
                                            (64, 512, 1000), (65, 33, 257), (200, 1111, 130),
                                            (2_000, 96, 2_100), (300, 2_048, 1_000),
                                            (1_500, 200, 1_704), (700, 1_024, 2_104),
                                            (40, 1_001, 500), (17, 4_096, 64), (2, 16_384, 40),
                                            (1, 16_385, 40), (2, 1_000, 33)])
def test_linear(learn, dtype, tokens, dim, out):
    x = randn(tokens, dim, seed=32, dtype=dtype, scale=2.0)
    check_linear(learn, x, dtype, out, f"{dtype}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,pad", [(1, 3), (70, 3), (70, 16)])
def test_linear_strides(learn, dtype, tokens, pad):
    def wide(v):
        b = torch.full((v.shape[0], v.shape[1] + 2 * pad), torch.nan, dtype=v.dtype)
        b[:, pad:-pad] = v
        return b.cuda()[:, pad:-pad]

    check_linear(learn, randn(tokens, 60, seed=33, dtype=dtype), dtype, 90, f"{dtype}", wide)


@pytest.mark.parametrize("tokens", [3, 70])
@pytest.mark.parametrize("pad", [3, 16])
def test_what_is_beside_the_results_stays(learn, tokens, pad):
    """Outputs in the middle of wider buffers: what is around them is left as it was."""
    from paper_1503_08294_amd import gsn
    x = randn(tokens, 48, seed=51, dtype=BF16).cuda()
    q = torch.full((tokens + 2, 48 + 2 * pad), 99, dtype=torch.int8, device="cuda")
    s = torch.full((tokens + 2,), -7.0, device="cuda")
    gsn.gsn_quantise(x, q[1:-1, pad:-pad], s[1:-1])
    want_q, want_s = ref.quantise(x.cpu())
    assert torch.equal(q[1:-1, pad:-pad].cpu().long(), want_q)
    assert torch.equal(s[1:-1].cpu(), want_s) and (s[[0, -1]] == -7).all()
    q[1:-1, pad:-pad] = 99
    assert (q == 99).all()
    w, ws = learn.quantise(randn(90, 48, seed=52).cuda())
    y = torch.full((tokens + 2, 90 + 2 * pad), 5.0, dtype=BF16, device="cuda")
    p = gsn.gsn_linear_params(gsn.GSN_BF16, 48, 90, tokens)
    room = torch.empty(gsn.gsn_linear_quantised_workspace_bytes(p), dtype=torch.uint8,
                       device="cuda")
    gsn.gsn_linear_quantised(p, x, w, ws, y[1:-1, pad:-pad], room)
    want, tol = ref.linear_8bit(x.cpu(), w.cpu(), ws.cpu())
    close(y[1:-1, pad:-pad], want, tol, "y")
    y[1:-1, pad:-pad] = 5
    assert (y == 5).all()


def test_linear_largest_sums(learn):
    """All products of one sign at their largest: the sum is 127^2 dim, and 2^14 dim for weights of
    -128."""
    dim = (1 << 17) - 1
    x = torch.ones(3, dim, device="cuda")
    w = torch.full((70, dim), 127, dtype=torch.int8, device="cuda")
    w[1] = -128
    one = torch.ones(70, device="cuda")
    y = learn.linear_8bit(x, w, one).double().cpu()
    want = torch.full((3, 70), 127.0 * dim, dtype=torch.float64)
    want[:, 1] = -128.0 * dim
    want *= 127 * float(np.float32(1) / np.float32(127))
    close(y, want, want.abs() * 4 * ref.U, "largest")


def test_linear_no_tokens(learn):
    w, s = learn.quantise(randn(9, 20, seed=34).cuda())
    assert learn.linear_8bit(torch.zeros(0, 20, device="cuda"), w, s).shape == (0, 9)
    q, s = learn.quantise(torch.zeros(0, 20, device="cuda"))
    assert q.shape == (0, 20) and s.shape == (0,)


# ---------------------------------------------------------------- beyond 32 bits ----

def test_entropy_of_weights_beyond_32_bits(learn):
    """More than 2^32 elements of w: the last classes' logits and gradients."""
    tokens, dim, classes = 3, 2_048, (1 << 21) + 70
    g = torch.Generator(device="cuda").manual_seed(35)
    w = torch.zeros(classes, dim, dtype=BF16, device="cuda")
    far = torch.randn(200, dim, generator=g, device="cuda").mul_(0.03).to(BF16)
    w[-200:] = far
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(BF16)
    t = torch.tensor([classes - 1, classes - 150, 5], dtype=torch.int32, device="cuda")
    loss, stats = learn.cross_entropy_forward(x, w, t)
    # the other classes' logits are 0
    l = x.double() @ far.double().t()
    total = torch.exp(l).sum(1) + (classes - 200)
    chosen = torch.stack([l[0, 199], l[1, 50], l[2, 0] * 0])
    want = torch.log(total) - chosen
    # a sum of dim products for each logit (of the chosen one too), some roundings of the result
    tol = 3 * dim * ref.U * (x.double().abs() @ far.double().abs().t()).max(1)[0] + 1e-5
    close(loss, want.cpu(), tol.cpu(), "loss")
    dx, dw = learn.cross_entropy_backward(torch.ones(tokens, device="cuda"), x, w, t, None, stats)
    d = torch.exp(l) / total[:, None]
    d[0, 199] -= 1
    d[1, 50] -= 1
    v = d.t() @ x.double()
    close(dw[-200:], v.cpu(), 2.0 ** -7 * (d.abs().t() @ x.double().abs()).cpu() + 1e-12, "dw")
    first = dw[5].double().cpu()
    close(first, -x[2].double().cpu(), 2.0 ** -7 * x.double().abs().sum(0).cpu(), "dw of class 5")
    v = d @ far.double()
    close(dx, v.cpu(), 2.0 ** -7 * (d.abs() @ far.double().abs()).cpu() + 1e-9, "dx")


@pytest.mark.parametrize("tokens", [2, 130])
def test_linear_of_weights_beyond_32_bits(learn, tokens):
    dim, out = 4_096, (1 << 20) + 37
    w = torch.zeros(out, dim, dtype=torch.int8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(36)
    w[-50:] = torch.randint(-127, 128, (50, dim), generator=g, device="cuda", dtype=torch.int8)
    s = torch.rand(out, generator=g, device="cuda")
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(BF16)
    y = learn.linear_8bit(x, w, s)
    want, tol = ref.linear_8bit(x.cpu(), w[-50:].cpu(), s[-50:].cpu())
    close(y[:, -50:], want, tol, "last rows")
    assert (y[:, :-50] == 0).all()


# ---------------------------------------------------- streams, graphs, all together ----

def calls(learn):
    """Calls of every operator, each with inputs of its own."""
    x, w, t, valid, dloss = (v.cuda() for v in entropy_inputs(70, 48, 260, BF16, 40, shut=0.1,
                                                              lost=0.1))
    _, stats = learn.cross_entropy_forward(x, w, t, valid)
    h = [None if v is None else v.cuda() for v in entropy_inputs(3, 40, 500, F16, 41)]
    _, hs = learn.cross_entropy_forward(h[0], h[1], h[2])
    m = randn(3, 60, 90, seed=42).cuda()
    one = randn(1, 24, 40, seed=47).cuda()
    wq, ws = learn.quantise(randn(200, 48, seed=43).cuda())
    return [lambda: learn.cross_entropy_forward(x, w, t, valid),
            lambda: learn.cross_entropy(x[:1], w, t[:1], valid),
            lambda: learn.cross_entropy_backward(dloss, x, w, t, valid, stats),
            lambda: learn.cross_entropy_backward(h[4], h[0], h[1], h[2], None, hs),
            lambda: learn.orthogonalise(m),
            lambda: learn.orthogonalise(one),
            lambda: learn.orthogonal_step(m, m + 1, 2 * m, 0.1),
            lambda: learn.quantise(x),
            lambda: learn.linear_8bit(x, wq, ws),
            lambda: learn.linear_8bit(x[:1], wq, ws)]


def flat(r):
    return [v for v in (r if isinstance(r, tuple) else (r,))]


def same(a, b):
    return all(torch.equal(p.float().nan_to_num(7), q.float().nan_to_num(7))
               for p, q in zip(flat(a), flat(b)))


def test_results_repeat_bit_for_bit_and_on_other_streams(learn):
    fs = calls(learn)
    want = [f() for f in fs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in fs]
    got = []
    for f, s in zip(fs, streams):
        with torch.cuda.stream(s):
            got.append(f())
    torch.cuda.synchronize()
    for i, (a, b, f) in enumerate(zip(want, got, fs)):
        assert same(a, b), i
        assert same(a, f()), i


def test_recorded_graphs_replay(learn):
    """Each call in a graph of its own and all in one, replayed with eager work between."""
    fs = calls(learn)
    want = [f() for f in fs]
    torch.cuda.synchronize()
    graphs = []
    for group in [[i] for i in range(len(fs))] + [list(range(len(fs)))]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = [fs[i]() for i in group]
        graphs.append((graph, group, out))
    for _ in range(3):
        for graph, group, out in graphs:
            for r in out:
                for v in flat(r):
                    v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for i, r in zip(group, out):
                assert same(r, want[i]), i
            assert same(fs[group[0]](), want[group[0]])


def test_all_together(learn):
    """A model of local experts that answers with a unit, as it would be trained and served: norm,
    routing, experts, the loss over the units, updates of the weights, the head in 8 bits."""
    from paper_1503_08294_amd import mixture
    tokens, dim, hidden, experts, classes = 512, 64, 32, 4, 777
    x = randn(tokens, dim, seed=44).cuda()
    t = (x[:, :10].argmax(1) * 70 + 3).int()
    valid = torch.ones(classes, dtype=torch.uint8, device="cuda")
    valid[0] = 0
    gate = randn(experts, dim, seed=45, scale=0.1).cuda()
    w1 = randn(experts, 2 * hidden, dim, seed=46, scale=dim ** -0.5).cuda().requires_grad_()
    w2 = randn(experts, dim, hidden, seed=47, scale=hidden ** -0.5).cuda().requires_grad_()
    head = torch.zeros(classes, dim, device="cuda", requires_grad=True)
    momenta = [torch.zeros_like(p) for p in (w1, w2, head)]

    def features(w1, w2):
        n = mixture.layer_norm(x)
        ids, weights = mixture.route(n @ gate.t(), 2)
        return n + mixture.experts(n, ids, weights, w1, w2)

    def loss_of(w1, w2, head):
        return learn.cross_entropy(features(w1, w2), head, t, valid).mean()

    for step in range(3):
        loss = loss_of(w1, w2, head)
        assert torch.isfinite(loss)
        grads = torch.autograd.grad(loss, (w1, w2, head))
        # the gradients of the head against a difference along themselves
        with torch.no_grad():
            v = grads[2] / grads[2].norm()
            # (the loss is a mean of numbers near log 777 with errors of some 1e-6)
            h = 0.01
            slope = (loss_of(w1, w2, head + h * v) - loss_of(w1, w2, head - h * v)) / (2 * h)
            assert abs(slope - grads[2].norm()) <= 1e-4 + 0.02 * grads[2].norm()
            for p, g, m in zip((w1, w2, head), grads, momenta):
                learn.orthogonal_step(p, g, m, 0.02, out=(p, m))
    with torch.no_grad():
        f = features(w1, w2)
        y = learn.linear_8bit(f, *learn.quantise(head))
        want = f.double() @ head.double().t()
        # both sides rounded to half a step of 1 / 127 of their rows' largest values
        df = f.double().abs().amax(1, keepdim=True) / 254
        dh = head.double().abs().amax(1) / 254
        tol = df * head.double().abs().sum(1) + (f.double().abs() + df).sum(1, keepdim=True) * dh
        close(y, want.cpu(), (tol * 1.001 + 1e-6).cpu(), "the head in 8 bits")
