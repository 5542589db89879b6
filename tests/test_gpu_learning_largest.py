"""The learning calls at the ends of their ranges: tokens, classes, elements of a row, sides."""
import math

import pytest
import torch

import learning_reference as ref
from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_most_tokens(dtype):
    tokens, dim, classes = 1 << 24, 8, 70
    g = gen(1)
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(dtype)
    w = (torch.randn(classes, dim, generator=g, device="cuda") * 0.4).to(dtype)
    t = torch.randint(-1, classes, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.rand(tokens, generator=g, device="cuda")
    loss, stats = learning.cross_entropy_forward(x, w, t)
    dx, dw = learning.cross_entropy_backward(dloss, x, w, t, None, stats)
    some = torch.cat([torch.arange(300), torch.arange(0, tokens, 99_991),
                      torch.arange(tokens - 300, tokens)]).cuda()
    want = ref.cross_entropy(x[some].cpu(), w.cpu(), t[some].cpu(), None, dloss[some].cpu())
    for got, name in ((loss[some], "loss"), (dx[some], "dx")):
        assert ((got.double().cpu() - want[name]).abs() <= want[name + "_tol"]).all(), name
    total = torch.zeros(classes, dim, dtype=torch.float64, device="cuda")
    size, square = torch.zeros_like(total), torch.zeros_like(total)
    for i in range(0, tokens, 1 << 20):
        s = slice(i, i + (1 << 20))
        y = x[s].double()
        d = torch.softmax(y @ w.double().t(), 1)
        d.scatter_add_(1, t[s].long().clamp(min=0)[:, None], -torch.ones_like(d[:, :1]))
        d *= torch.where(t[s] >= 0, dloss[s].double(), 0.0)[:, None]
        total += d.t() @ y
        size += d.abs().t() @ y.abs()
        square += d.square().t() @ y.square()
    # gradients of logits are rounded to their type, each by itself: four standard deviations of half
    # a step (its deviation is its size by sqrt 3), 2^-16 of all for the logits' and exponentials'
    # own errors and for sums of some 2^15 terms a split; one rounding of the result
    u = torch.finfo(dtype).eps / 2
    tol = 4 * u * (square / 3).sqrt() + 2.0 ** -16 * size + u * total.abs()
    assert ((dw.double() - total).abs() <= tol).all()


def test_most_classes():
    """Two tokens, rows of one element: logits x w, all of the sums in the joins."""
    classes = 1 << 28
    g = gen(2)
    w = torch.randn(classes, 1, generator=g, device="cuda", dtype=BF16)
    x = torch.tensor([[0.5], [-2.0]], dtype=BF16, device="cuda")
    t = torch.tensor([classes - 1, 7], dtype=torch.int32, device="cuda")
    loss, stats = learning.cross_entropy_forward(x, w, t)
    total = torch.zeros(2, dtype=torch.float64, device="cuda")
    for i in range(0, classes, 1 << 24):
        total += torch.exp(w[i:i + (1 << 24)].double() * x.double().t()).sum(0)
    chosen = x[:, 0].double() * w[t.long(), 0].double()
    want = total.log() - chosen
    # a thread joins 2^14 parts, one after the other, each with an exponential or two and a sum
    assert ((loss.double() - want).abs() <= (1 << 14) * 4 * U + 16 * U * want).all()
    dx, dw = learning.cross_entropy_backward(torch.ones(2, device="cuda"), x, w, t, None, stats)
    for i in [0, 1 << 27, classes - (1 << 16)]:
        s = slice(i, i + (1 << 16))
        d = torch.exp(w[s].double() * x.double().t()) / total
        for token, c in enumerate(t.tolist()):
            if s.start <= c < s.stop:
                d[c - s.start, token] -= 1
        want = d @ x.double()
        tol = (2.0 ** -8 + (1 << 14) * 4 * U + 2.0 ** -15) * (d.abs() @ x.double().abs())
        assert ((dw[s].double() - want).abs() <= tol).all()


def test_most_tokens_of_a_layer():
    tokens = 1 << 24
    g = gen(3)
    x = torch.randn(tokens, 16, generator=g, device="cuda", dtype=BF16)
    w, scales = learning.quantise(torch.randn(24, 16, generator=g, device="cuda"))
    y = learning.linear_8bit(x, w, scales)
    some = torch.cat([torch.arange(0, tokens, 99_991), torch.arange(tokens - 300, tokens)]).cuda()
    want, tol = ref.linear_8bit(x[some].cpu(), w.cpu(), scales.cpu())
    assert ((y[some].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_longest_rows_in_8_bits(dtype):
    dim = 1 << 27
    x = torch.randn(2, dim, generator=gen(4), device="cuda").to(dtype)
    x[1, -1] = 100
    q, s = learning.quantise(x)
    for r in range(2):
        top = x[r].float().abs().max()
        assert s[r].item() == (top.cpu() / torch.tensor(127.0)).item()
        for part in (slice(0, 1 << 16), slice(dim - (1 << 16), dim)):
            assert torch.equal(q[r, part].double(), torch.round(x[r, part].double() / s[r].double()))


def test_longest_sides():
    """One step: a x + (b A + c A A) x of some rows, A of all of them."""
    side = 1 << 15
    a, b, c = learning.COEFFICIENTS
    x = torch.randn(side, side, generator=gen(5), device="cuda")
    got = learning.orthogonalise(x, steps=1)
    norm = math.sqrt(sum(v.double().square().sum().item() for v in x.split(1 << 12))) + 1e-7
    rows = torch.tensor([0, 1, 63, 64, 127, 128, 16_383, 16_384, side - 129, side - 1]).cuda()

    def by(m, transposed):  # of some rows m, with x / norm or its transpose, in 64 bits
        if transposed:
            return torch.cat([m @ (v.double() / norm).t() for v in x.split(1 << 12)], 1)
        return sum(m[:, i:i + (1 << 12)] @ (x[i:i + (1 << 12)].double() / norm)
                   for i in range(0, side, 1 << 12))

    start = x[rows].double() / norm
    ax = by(by(start, True), False)          # rows of A x
    want = a * start + b * ax + c * by(by(ax, True), False)
    # a row is off by 22 bits of it twice (2^-21) and by the roundings of its sums, 4 sqrt(3 side) U
    # of it: the polynomial is within a tenth of a for singular values of at most 2 / sqrt(side)
    tol = (2.0 ** -21 + 4 * math.sqrt(3 * side) * U) * 1.1 * want.norm(dim=1)
    assert ((got[rows].double() - want).norm(dim=1) <= tol).all()
