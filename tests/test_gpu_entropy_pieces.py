"""The cross entropy over classes that a pass takes in several pieces (512 MB of the copy of w or of
the logits' gradients, 256 MB of a forward pass's parts): sums carried from piece to piece, targets
in early and late ones, copies made anew, and the sizes at which a path ends."""
import pytest
import torch

import learning_reference as ref
from paper_1503_08294_amd import gsn, learning

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24


def randn(*shape, g, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def logit_error(x, w):
    """Of each token's logits: a sum of dim products makes dim roundings at most, each of a partial
    sum that is below |x| |w|; independent ones, four of their standard deviations (half a step has
    the deviation U / sqrt 3): 4 sqrt(dim / 3) U |x| |w|.  Of 22 bits of an element 8 U |x| |w| more,
    and 2^-24 of those that they have no room for."""
    return (4 * (w.shape[1] / 3) ** 0.5 + 8) * U * x.norm(dim=1) * w.norm(dim=1).max() + U


def formulas(x, w, t, valid, dloss, some):
    """Losses and dx of the tokens `some`, dw of all tokens, in 64 bits, and their tolerances: a logit
    is off by E (logit_error()), a probability by (4 E + (far + 6) 2 U + (64 + classes / 64) 2 U) of
    itself, where far is how far its logit is below the largest; a gradient of a logit by that and
    half a step of its type (of float16 2^-39 of the largest dloss besides), a result by a rounding
    a term and half a step of its own."""
    u = torch.finfo(x.dtype).eps / 2
    classes, dim = w.shape
    there = torch.ones(classes, dtype=torch.bool, device="cuda") if valid is None else valid != 0
    live = t >= 0
    w = torch.where(there[:, None], w.double(), 0.0)
    x = torch.where(live[:, None], x.double(), 0.0)
    g = torch.where(live, dloss.double(), 0.0)
    loss, loss_tol = torch.zeros_like(g), torch.zeros_like(g)
    dx, dx_tol = torch.zeros_like(x[some]), torch.zeros_like(x[some])
    dw, dw_tol = torch.zeros_like(w), torch.zeros_like(w)
    place = {int(v): i for i, v in enumerate(some.tolist())}
    most = g.abs().max()
    for i in range(0, len(x), 20_000):
        s = slice(i, i + 20_000)
        logits = (x[s] @ w.t()).masked_fill(~there, -torch.inf)
        e = logit_error(x[s], w)[:, None]
        logp = logits.log_softmax(1)
        p = logp.exp()
        at = t[s].long().clamp(min=0)[:, None]
        far = (logits.max(1, keepdim=True)[0] - logits).masked_fill(~there, 0.0)
        rel = 4 * e + (far + 6) * 2 * U + (64 + classes / 64) * 2 * U
        loss[s] = torch.where(live[s], -logp.gather(1, at)[:, 0], 0.0)
        loss_tol[s] = 4 * e[:, 0] + (p * rel).sum(1) + 8 * U * (
            loss[s].abs() + logits.logsumexp(1).abs() + 1)
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        d = (p - one) * g[s, None]
        off = (p * rel + 4 * U * one) * g[s, None].abs() + u * d.abs() + 2.0 ** -130
        if u == 2.0 ** -11:
            off = off + 2.0 ** -39 * most
        off = off * there * live[s, None]
        dw += d.t() @ x[s]
        dw_tol += (off + 32 * U * d.abs()).t() @ x[s].abs()
        mine = [j for j in some.tolist() if i <= j < i + 20_000]
        if mine:
            rows = torch.tensor(mine, device="cuda") - i
            to = [place[j] for j in mine]
            dx[to] = d[rows] @ w
            dx_tol[to] = (off[rows] + 32 * U * d[rows].abs()) @ w.abs()
    dx_tol += u * dx.abs() + 2.0 ** -25
    dw_tol += u * dw.abs() + 2.0 ** -25
    return loss, loss_tol, dx, dx_tol, dw, dw_tol


def check(x, w, t, valid, dloss, every):
    loss, stats = learning.cross_entropy_forward(x, w, t, valid)
    dx, dw = learning.cross_entropy_backward(dloss, x, w, t, valid, stats)
    some = torch.arange(0, len(x), every, device="cuda")
    want = formulas(x, w, t, valid, dloss, some)
    for got, v, tol, name in ((loss, *want[:2], "loss"), (dx[some], *want[2:4], "dx"),
                              (dw, *want[4:], "dw")):
        assert torch.isfinite(got).all(), name
        over = ((got.double() - v).abs() - tol).max()
        assert over <= 0, f"{name}: {over} beyond the tolerance"


def inputs(tokens, dim, classes, dtype, seed, shut, lost=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = randn(classes, dim, g=g, dtype=dtype, scale=dim ** -0.5)
    x = randn(tokens, dim, g=g, dtype=dtype)
    t = torch.randint(0, classes, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    t[:2] = torch.tensor([0, classes - 1])
    t[torch.rand(tokens, generator=g, device="cuda") < lost] = -1
    valid = None
    if shut:
        valid = (torch.rand(classes, generator=g, device="cuda") >= shut).to(torch.uint8)
        valid[t[t >= 0].long()] = 1
        w[valid == 0] = torch.nan
    x[t < 0] = torch.nan
    dloss = torch.rand(tokens, generator=g, device="cuda") + 0.5
    return x, w, t, valid, dloss / tokens


# wide rows: pieces of 512 MB of w.  dim 65,536 in 2 bytes: 4,096 classes a piece, 65,001 in 4 bytes
# 2,048
@pytest.mark.parametrize("dtype,tokens,dim,classes,shut", [
    (BF16, 100, 65_536, 4_500, 0.0), (BF16, 70, 65_001, 4_300, 0.1),
    (F16, 1_030, 65_536, 8_300, 0.05), (F32, 300, 65_001, 4_200, 0.1),
    (F32, 300, 65_536, 4_200, 0.0), (F32, 1_030, 65_536, 3_000, 0.1),
    (F32, 60, 65_001, 3_000, 0.1)])
def test_wide_rows(dtype, tokens, dim, classes, shut):
    check(*inputs(tokens, dim, classes, dtype, tokens + classes, shut), every=7)


# many tokens: pieces of 256 MB of parts forward, of 512 MB of gradients backward.  300,000 tokens:
# 7,168 classes a piece forward, 768 backward in 2 bytes and 256 in 4; 600,000: 3,328 and 256
@pytest.mark.parametrize("dtype,tokens,dim,classes,shut", [
    (BF16, 600_000, 16, 3_500, 0.1), (F16, 600_000, 17, 3_400, 0.0), (F16, 300_000, 33, 1_000, 0.1),
    (F32, 300_000, 17, 700, 0.1), (F32, 600_000, 8, 3_400, 0.05)])
def test_many_tokens(dtype, tokens, dim, classes, shut):
    check(*inputs(tokens, dim, classes, dtype, dim + classes, shut), every=9_973)


def test_pieces_of_both_kinds():
    """Binary32: a piece whose rows hold a number far larger than the others, which shuts classes
    out for odd tokens and are the targets of the even ones, beside pieces whose rows do not."""
    x, w, t, _, _ = inputs(300, 65_536, 4_200, F32, 5, 0.0, lost=0.0)
    odd = torch.arange(300, device="cuda") % 2 == 1
    x[:, -1], w[:, -1] = odd.float(), 0.0
    w[3_000:3_100, -1] = -1e9  # (of the second piece of three)
    t = torch.where(odd, t % 3_000, 3_000 + t % 100)
    loss = learning.cross_entropy(x, w, t)
    logits = x.double() @ w.double().t()
    want = -logits.log_softmax(1).gather(1, t.long()[:, None])[:, 0]
    w[:, -1] = 0  # (what is shut out has no part)
    tol = 5 * logit_error(x.double(), w.double()) + 1e-5
    assert tol.max() < 0.1
    assert ((loss.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("tokens", [16, 17, 32, 33, 64, 65, 255, 256, 257, 1_024, 1_025])
@pytest.mark.parametrize("dim", [40, 41])
def test_where_a_path_ends(dtype, tokens, dim):
    """Few rows, gradients in two values, logits in two values, joins: the last size of each and the
    first of the next, rows at multiples of 16 bytes and others."""
    x, w, t, valid, dloss = inputs(tokens, dim, 130, dtype, tokens, 0.1)
    want = ref.cross_entropy(x.cpu(), w.cpu(), t.cpu(), valid.cpu(), dloss.cpu())
    loss, stats = learning.cross_entropy_forward(x, w, t, valid)
    dx, dw = learning.cross_entropy_backward(dloss, x, w, t, valid, stats)
    for got, name in ((loss, "loss"), (dx, "dx"), (dw, "dw")):
        assert ((got.double().cpu() - want[name]).abs() <= want[name + "_tol"]).all(), name


def test_the_sizes_take_pieces():
    """What the cases above are for: a workspace that holds all classes' copies, parts or gradients
    would be larger."""
    def size(dtype, dim, classes, tokens, backward):
        return gsn.gsn_cross_entropy_workspace_bytes(
            gsn.gsn_entropy_params(dtype, dim, classes, tokens), backward)

    assert size(gsn.GSN_BF16, 65_536, 1 << 20, 100, False) < 2 * 65_536 << 20
    assert size(gsn.GSN_BF16, 65_536, 4_096, 100, False) > 65_536 * 4_096 * 2
    assert size(gsn.GSN_BF16, 65_536, 8_192, 100, False) < 65_536 * 8_192 * 2
    for sizes, tokens, backward in (((65_536, 4_200), 300, True), ((65_536, 3_000), 1_030, False)):
        assert size(gsn.GSN_F32, *sizes, tokens, backward) <= 1.1 * size(gsn.GSN_F32, 65_536, 2_048,
                                                                         tokens, backward)
    assert size(gsn.GSN_BF16, 16, 3_500, 600_000, False) <= 1.01 * size(gsn.GSN_BF16, 16, 3_328,
                                                                        600_000, False)
