"""Numbers at the ends of binary32 in the learning calls: matrices of tiny and of huge norms, tokens
whose dloss is not finite."""
from __future__ import annotations

import pytest
import torch

from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu

SIZES = ((33, 70), (70, 33), (200, 312), (312, 200))  # in one workgroup each, and in tiles


def _whole(rows, cols, seed):
    """Whole numbers: times a power of two they are the same binary32 values, subnormal too."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-8, 9, (2, rows, cols), generator=g).float().cuda()


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("power", (-145, -130, -110, -60, 60, 110, 123))
def test_a_matrix_times_a_power_of_two_is_the_same_one(rows, cols, power):
    x = _whole(rows, cols, 5)
    half = power // 2  # (2^-145 itself is no normal number)
    scaled = x * 2.0 ** half * 2.0 ** (power - half)
    want = learning.orthogonalise(x, eps=0.0)
    got = learning.orthogonalise(scaled, eps=0.0)
    torch.cuda.synchronize()
    assert torch.isfinite(want).all() and want.abs().max() > 0.01
    assert torch.equal(got, want)
    # an update by the gradient alone
    zeros = torch.zeros_like(x)
    for w in (torch.float32, torch.bfloat16):
        if w == torch.bfloat16 and not -120 <= power <= 120:
            continue
        a, b = (learning.orthogonal_step(zeros.to(w), v.to(w), zeros, 1.0, beta=0.0,
                                         nesterov=False, eps=0.0)[0] for v in (x, scaled))
        torch.cuda.synchronize()
        assert torch.equal(a, b) and a.abs().max() > 0.01


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("tokens", (17, 130))
@pytest.mark.parametrize("value", (torch.inf, -torch.inf, torch.nan))
def test_a_dloss_that_is_not_finite_is_its_own_tokens_matter(dtype, tokens, value):
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, 72, generator=g).to(dtype).cuda()
    w = torch.randn(301, 72, generator=g).to(dtype).cuda()
    targets = torch.randint(0, 301, (tokens,), generator=g, dtype=torch.int32).cuda()
    dloss = torch.rand(tokens, generator=g).cuda()
    stats = learning.cross_entropy_forward(x, w, targets)[1]
    other = targets.clone()
    other[5] = -1
    want = learning.cross_entropy_backward(dloss, x, w, other, None, stats)[0]
    dloss[5] = value
    got = learning.cross_entropy_backward(dloss, x, w, targets, None, stats)[0]
    torch.cuda.synchronize()
    rest = torch.arange(tokens, device="cuda") != 5
    assert torch.equal(got[rest], want[rest]) and torch.isfinite(got[rest]).all()
    assert not torch.isfinite(got[5].float()).any()


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("tokens,classes,dim", [(1, 300, 64), (3, 1001, 72), (17, 70, 131),
                                                (32, 5003, 96), (31, 129, 40)])
def test_gradients_of_few_tokens_are_rounded_once(dtype, tokens, classes, dim):
    """Results differ from the formulas' by their own rounding, and by what binary32 sums and second
    values leave: 2 u^2 of a gradient of the logits (u half a step), and twice the logits' error
    (dim 2^-24 sum |x w|), exp's (|l - largest| + 3) 2^-23 and the sums' 2^-24 an addition of it."""
    u, one = torch.finfo(dtype).eps / 2, 2.0 ** -24
    g = torch.Generator().manual_seed(tokens + classes)
    w = (torch.randn(classes, dim, generator=g) * dim ** -0.5).to(dtype)
    t = torch.randint(0, classes, (tokens,), generator=g, dtype=torch.int32)
    x = (torch.randn(tokens, dim, generator=g)
         + 4 * torch.rand(tokens, 1, generator=g) * w[t.long()].float()).to(dtype)
    dloss = torch.rand(tokens, generator=g) + 0.5
    stats = learning.cross_entropy_forward(x.cuda(), w.cuda(), t.cuda())[1]
    dx, dw = learning.cross_entropy_backward(dloss.cuda(), x.cuda(), w.cuda(), t.cuda(), None,
                                             stats)
    x, w, scale = x.double(), w.double(), dloss.double()[:, None]
    logits = x @ w.t()
    p = logits.softmax(1)
    d = p.clone()
    d[torch.arange(tokens), t.long()] -= 1
    far = (logits.max(1, keepdim=True)[0] - logits).max(1, keepdim=True)[0]
    rel = 4 * dim * one * (x.abs() @ w.abs().t()).max(1, keepdim=True)[0] \
        + (2 * far + 6 + 64 + classes / 64 + 8) * 2 * one
    step = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    kept = 2 * u * u * d.abs() + rel * p + (step * 2.0 ** -14 if dtype == torch.float16 else step)
    for got, a, b, e in ((dx, d * scale, w, kept * scale),
                         (dw, (d * scale).t(), x, (kept * scale).t())):
        want = a @ b
        tol = (e + (a.shape[1] + 12) * one * a.abs()) @ b.abs()
        tol = (tol + u * (want.abs() + tol)) + step
        assert ((got.double().cpu() - want).abs() <= tol).all()
