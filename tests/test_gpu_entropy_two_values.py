"""The cross entropy of so many tokens in binary32 that its logits are made of two float16 values:
masks, strides, sizes of tiles, numbers that are not finite, streams and graphs."""
import pytest
import torch

import learning_reference as ref
from paper_1503_08294_amd import learning
from test_gpu_learning import check_entropy, close, entropy_inputs, flat, same

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.mark.parametrize("tokens,dim,classes", [
    (256, 1, 1), (256, 1, 3), (257, 3, 2), (300, 40, 90), (260, 129, 65), (511, 64, 64),
    (513, 33, 257), (1_025, 17, 300), (1_300, 250, 1_100), (4_100, 72, 2_100), (260, 1_100, 5_000)])
def test_sizes(tokens, dim, classes):
    check_entropy(learning, *entropy_inputs(tokens, dim, classes, F32, 1, shut=0.02, lost=0.02),
                  f"{tokens}")


@pytest.mark.parametrize("tokens,dim,classes", [(256, 16, 40), (300, 65, 200), (1_100, 64, 300)])
@pytest.mark.parametrize("value", [torch.nan, torch.inf, -torch.inf, 3e38])
def test_masks(tokens, dim, classes, value):
    x, w, t, valid, dloss = entropy_inputs(tokens, dim, classes, F32, 2, shut=0.3, lost=0.2)
    t[0] = classes + 3
    t[1:3] = torch.tensor([2 ** 31 - 1, -2 ** 31])
    valid[t[3]] = 0
    lost = (t < 0) | (t >= classes)
    lost |= valid[t.clamp(0, classes - 1).long()] == 0
    x[lost], w[valid == 0], dloss[lost] = value, value, torch.nan
    dx, dw = check_entropy(learning, x, w, t, valid, dloss, f"{value}")
    assert (dx[lost.cuda()] == 0).all() and (dw[valid.cuda() == 0] == 0).all()


@pytest.mark.parametrize("dim", [24, 33])
def test_nothing(dim):
    """Every class shut, no token with a target, rows of zeros."""
    x, w, t, _, dloss = entropy_inputs(300, dim, 30, F32, 3)
    check_entropy(learning, x, w, t, torch.zeros(30, dtype=torch.uint8), dloss, "no class")
    check_entropy(learning, x, w, torch.full_like(t, -5), None, dloss, "no target")
    check_entropy(learning, x * 0, w, t, None, dloss, "tokens of zeros")
    check_entropy(learning, x, w * 0, t, None, dloss, "classes of zeros")


@pytest.mark.parametrize("dim,pad", [(64, 1), (64, 4), (33, 7), (40, 24)])
def test_strides(dim, pad):
    def wide(v):
        b = torch.full((v.shape[0], v.shape[1] + 2 * pad), torch.nan)
        b[:, pad:-pad] = v
        return b.cuda()[:, pad:-pad]

    check_entropy(learning, *entropy_inputs(270, dim, 150, F32, 4), f"{dim}", wide)


@pytest.mark.parametrize("times", [1, 60, 400])
def test_large_logits(times):
    """Logits of some hundreds and thousands; the largest are made in binary32."""
    x, w, t, _, dloss = entropy_inputs(300, 64, 90, F32, 5)
    x[:10] *= times
    x[10] = 50 * w[t[10].long()]
    dloss[11] *= 2.0 ** -18
    dloss[12] = 0
    check_entropy(learning, x, w, t, None, dloss, f"{times}")


@pytest.mark.parametrize("value", [torch.inf, -torch.inf, torch.nan])
@pytest.mark.parametrize("where", ["x", "dloss"])
def test_a_token_that_is_not_finite_is_its_own_matter(value, where):
    x, w, t, _, dloss = (v if v is None else v.cuda() for v in entropy_inputs(300, 72, 301, F32, 6))
    want, stats = learning.cross_entropy_forward(x, w, t)
    want_dx = learning.cross_entropy_backward(dloss, x, w, t, None, stats)[0]
    (x if where == "x" else dloss)[5] = value
    loss, stats = learning.cross_entropy_forward(x, w, t)
    dx = learning.cross_entropy_backward(dloss, x, w, t, None, stats)[0]
    rest = torch.arange(300, device="cuda") != 5
    # (with x the others' logits are made in binary32: both are within their tolerances)
    host = [v.cpu() for v in (x, w, t, dloss)]
    tol = ref.cross_entropy(host[0][rest.cpu()], host[1], host[2][rest.cpu()], None,
                            host[3][rest.cpu()])
    assert ((loss - want).double().cpu().abs()[rest.cpu()] <= 2 * tol["loss_tol"]).all()
    assert ((dx - want_dx).double().cpu().abs()[rest.cpu()] <= 2 * tol["dx_tol"]).all()
    assert not torch.isfinite(dx[5]).any()
    if where == "x":
        assert not torch.isfinite(loss[5])


def test_streams_and_graphs():
    """The same bits alone, on other streams at a time, and from a graph's replays with eager work
    between; of logits in two values and of rows that have none of them."""
    cases = []
    for seed, last in ((7, 0.0), (8, -1e9)):
        x, w, t, valid, dloss = (v.cuda() for v in entropy_inputs(300, 48, 260, F32, seed, shut=0.1))
        w[20:30, -1] = last
        cases.append((x, w, t, valid, dloss, learning.cross_entropy_forward(x, w, t, valid)[1]))
    fs = [f for x, w, t, valid, dloss, stats in cases for f in (
        lambda x=x, w=w, t=t, valid=valid: learning.cross_entropy_forward(x, w, t, valid),
        lambda x=x, w=w, t=t, valid=valid, dloss=dloss, stats=stats:
        learning.cross_entropy_backward(dloss, x, w, t, valid, stats))]
    want = [f() for f in fs]
    torch.cuda.synchronize()
    got = []
    for f, s in zip(fs, [torch.cuda.Stream() for _ in fs]):
        with torch.cuda.stream(s):
            got.append(f())
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [f() for f in fs]
    for i in range(4):
        for r in out:
            for v in flat(r):
                v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(out, want))
        assert same(fs[i](), want[i])


def test_losses_alone_are_those_with_statistics():
    x, w, t, valid, _ = (v.cuda() for v in entropy_inputs(700, 60, 1_000, F32, 9, shut=0.1))
    loss = learning.cross_entropy(x, w, t, valid)
    assert torch.equal(loss, learning.cross_entropy_forward(x, w, t, valid)[0])
    # tokens do not depend on each other
    half = learning.cross_entropy(x[:350], w, t[:350], valid)
    want = ref.cross_entropy(x[:350].cpu(), w.cpu(), t[:350].cpu(), valid.cpu())
    close(half, want["loss"], want["loss_tol"], "half")
