"""Logits in binary32 where a row holds a number far larger than the others: a feature whose
weights shut classes out by a large negative number, or by an infinity, for some tokens and not for
others."""
import pytest
import torch

from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def inputs(tokens, dim, classes, value, seed):
    """The last feature is 1 for every other token, for which `value` shuts out half of the classes;
    it is 0 for the rest."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, dim, generator=g)
    w = torch.randn(classes, dim, generator=g) * 0.3
    x[:, -1] = torch.arange(tokens) % 2
    w[:, -1] = torch.where(torch.arange(classes) % 2 == 1, value, 0.0)
    t = 2 * torch.randint(0, classes // 2, (tokens,), generator=g).int()
    return x, w, t


def tolerance(x, w, logits):
    """A logit is off by (dim + 8) U sum |x w| (22 bits of each, or binary32), and by 2^-24 where 22
    bits do not reach; the sum of the exponentials by their errors, at most (far + 3) 2 U each and U
    an addition; the loss by three roundings of numbers near itself."""
    dim, classes = x.shape[1], w.shape[0]
    keep = w.abs() < 1e6  # (what is shut out has no part)
    size = (x.abs() @ (w * keep).abs().t()).max(1)[0]
    e = (dim + 8) * U * size + U
    p = logits.softmax(1)
    far = logits.max(1, keepdim=True)[0] - logits
    far = torch.where(p > 0, far, 0.0)
    total = (64 + classes / 64) * U + (p * (far + 3)).sum(1) * 2 * U
    near = logits.logsumexp(1).abs() + logits.abs().where(p > 0, 0.0).max(1)[0] + 1
    return 4 * e + total + 8 * U * near


# (few tokens are multiplied in binary32; parts of 1,100 are joined by another kernel)
@pytest.mark.parametrize("tokens", [30, 160, 192, 255, 256, 300, 1_100])
@pytest.mark.parametrize("value", [-1e4, -1e9, -1e30, -torch.finfo(torch.float32).max])
@pytest.mark.parametrize("dim,classes", [(32, 120), (37, 701)])
def test_a_feature_that_shuts_classes_out(tokens, value, dim, classes):
    x, w, t = inputs(tokens, dim, classes, value, tokens + dim)
    loss, stats = learning.cross_entropy_forward(x.cuda(), w.cuda(), t.cuda())
    logits = x.double() @ w.double().t()
    want = torch.nn.functional.cross_entropy(logits, t.long(), reduction="none")
    tol = tolerance(x.double(), w.double(), logits)
    assert ((loss.double().cpu() - want).abs() <= tol).all()
    # the gradient of a class that is shut out for a token has no part of that token
    dx, dw = learning.cross_entropy_backward(torch.ones(tokens, device="cuda"), x.cuda(), w.cuda(),
                                             t.cuda(), None, stats)
    d = logits.softmax(1)
    d[torch.arange(tokens), t.long()] -= 1
    want = d.t() @ x.double()
    # (a probability is off by twice the tolerance of its loss)
    off = (d.abs() * 2 * tol[:, None] + 4 * U * d.abs() + 4 * U).t() @ x.double().abs() \
        + (tokens + 12) * U * (d.abs().t() @ x.double().abs()) + U * want.abs()
    got = dw.double().cpu()
    assert ((got - want).abs() <= off).all()
    assert torch.isfinite(dx).all()


@pytest.mark.parametrize("tokens", [30, 160, 192, 256, 300, 1_100])
def test_an_infinity_that_shuts_classes_out(tokens):
    """(For every token: an infinity by 0 is NaN.)"""
    x, w, t = inputs(tokens, 32, 120, -torch.inf, tokens)
    x[:, -1] = 1
    loss = learning.cross_entropy(x.cuda(), w.cuda(), t.cuda())
    logits = x.double() @ w.double().t()
    assert torch.isinf(logits[:, 1::2]).all()
    logits = logits[:, ::2]
    want = torch.nn.functional.cross_entropy(logits, t.long() // 2, reduction="none")
    tol = tolerance(x.double(), w.double()[::2], logits)
    assert ((loss.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("tokens", [160, 192, 300])
def test_rows_that_are_not_there_may_hold_anything(tokens):
    """Tokens without a target and classes that are not valid do not change what the others get, bit
    for bit."""
    x, w, t = inputs(tokens, 32, 120, -1.0, 3)
    valid = torch.ones(120, dtype=torch.uint8)
    valid[5::9] = 0
    valid[t.long()] = 1
    t[7::10] = -1
    got = []
    for value in (0.0, 1e30, torch.inf, torch.nan):
        y, v = x.clone(), w.clone()
        y[7::10], v[valid == 0] = value, value
        loss, stats = learning.cross_entropy_forward(y.cuda(), v.cuda(), t.cuda(), valid.cuda())
        dx, dw = learning.cross_entropy_backward(torch.ones(tokens, device="cuda"), y.cuda(),
                                                 v.cuda(), t.cuda(), valid.cuda(), stats)
        got.append((loss, dx, dw))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
