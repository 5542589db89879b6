"""Logits of binary32 rows whose sizes multiply to more, or less, than binary32 holds."""
import math

import pytest
import torch

from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [5, 159, 160, 255, 256, 300])
@pytest.mark.parametrize("power", [60, 70, 100, 127])
def test_large_rows_that_are_orthogonal(tokens, power):
    """A token and a class that are large where the other is zero: their logit is 0, and with the
    other classes' logits 0 as well the token's loss is the logarithm of the number of classes, in
    binary32 within 4 roundings."""
    g = torch.Generator().manual_seed(tokens)
    classes = 90
    x, w = torch.randn(tokens, 8, generator=g), torch.randn(classes, 8, generator=g)
    x[:, 6] = w[:, 7] = 0
    x[2] = 0
    x[2, 7] = 2.0 ** power
    w[3, 6] = -2.0 ** power
    t = torch.randint(0, classes, (tokens,), generator=g, dtype=torch.int32)
    loss, stats = learning.cross_entropy_forward(x.cuda(), w.cuda(), t.cuda())
    assert torch.isfinite(loss).all()
    assert abs(loss[2].item() - math.log(classes)) <= 4 * 2.0 ** -24 * math.log(classes)
    # the gradient of a logit of token 2 is 1 / classes, and that less 1 for its target
    dx, dw = learning.cross_entropy_backward(torch.ones(tokens, device="cuda"), x.cuda(), w.cuda(),
                                             t.cuda(), None, stats)
    want = torch.full((classes,), 2.0 ** power / classes, dtype=torch.float64)
    want[t[2]] -= 2.0 ** power
    got = dw[:, 7].double().cpu()
    assert ((got - want).abs() <= 8 * 2.0 ** -24 * 2.0 ** power).all()
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("tokens", [5, 160, 256, 300])
def test_a_large_row_by_a_small_one(tokens):
    """Rows of 2^100 by rows of 2^-100: the logits are those of the rows themselves."""
    g = torch.Generator().manual_seed(tokens)
    x, w = torch.randn(tokens, 24, generator=g), torch.randn(70, 24, generator=g)
    t = torch.randint(0, 70, (tokens,), generator=g, dtype=torch.int32).cuda()
    want = learning.cross_entropy(x.cuda(), w.cuda(), t)
    for power in (100, -100):
        got = learning.cross_entropy((x * 2.0 ** power).cuda(), (w * 2.0 ** -power).cuda(), t)
        # (powers of two change no digit, but for those that 2^-100 leaves no room for)
        assert ((got - want).abs() <= 1e-5).all()


@pytest.mark.parametrize("tokens", [5, 160, 256, 300])
@pytest.mark.parametrize("power", [-120, -110, 110, 120])
def test_rows_near_both_ends_of_binary32(tokens, power):
    """The logits of x times 2^power and w times 2^-power, all of them normal numbers, are those of x
    and w, and so are the losses; each is off by dim + 8 roundings of a logit's sum of magnitudes,
    below 24 x 3, and as many of its own."""
    g = torch.Generator().manual_seed(tokens)
    x, w = (torch.rand(n, 24, generator=g) + 0.5 for n in (tokens, 70))
    x *= torch.randint(0, 2, x.shape, generator=g) * 2 - 1
    w *= torch.randint(0, 2, w.shape, generator=g) * 2 - 1
    t = torch.randint(0, 70, (tokens,), generator=g, dtype=torch.int32).cuda()
    want = torch.nn.functional.cross_entropy(x.double() @ w.double().t(), t.long().cpu(),
                                             reduction="none")
    y, v = x * 2.0 ** power, w * 2.0 ** -power
    assert y.abs().min() >= 2.0 ** -126 and v.abs().min() >= 2.0 ** -126
    got = learning.cross_entropy(y.cuda(), v.cuda(), t).double().cpu()
    assert ((got - want).abs() <= 3 * 32 * 2.0 ** -24 * 72).all()
