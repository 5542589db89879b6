"""The experts' products in tiles of 256 x 256 at sizes where a sum ends early: of one stage of k,
of two, and of less than one; where blocks end early; and with tokens past 2^32 elements."""
import pytest
import torch

from test_gpu_mixture import (BF16, F16, expert_inputs, expert_tolerance, experts_in_float64,
                              far_apart, near)

pytestmark = pytest.mark.gpu

NAMES = ("out", "dx", "dweights", "dw1", "dw2")


@pytest.fixture(scope="module")
def mix():
    from paper_1503_08294_amd import mixture
    return mixture


# (a stage is 64 of k; 128 tiles of the first product and more take sides of 256)
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,experts,k,dim,hidden", [
    (16_384, 8, 2, 64, 512), (16_384, 8, 2, 512, 64), (17_001, 4, 2, 520, 32),
    (17_001, 4, 2, 56, 264), (17_001, 4, 2, 8, 8), (9_001, 4, 2, 72, 520), (17_001, 4, 2, 264, 72)])
def test_sums_of_few_stages(mix, dtype, tokens, experts, k, dim, hidden):
    a = [t.cuda() for t in expert_inputs(dtype, tokens, experts, k, dim, hidden, 61)]
    x, ids, weights, w1, w2, dout = a
    ids[5], ids[6, 0] = -1, experts
    want = experts_in_float64(*a)
    rel = expert_tolerance(dtype, dim, hidden, tokens * k)
    first = None
    for _ in range(3):
        out, saved = mix.experts_forward(x, ids, weights, w1, w2)
        got = (out, *mix.experts_backward(dout, x, ids, weights, w1, w2, saved))
        for g, v, name in zip(got, want, NAMES):
            near(g, v.detach().cpu(), rel, name)
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(got, first))
    near(mix.experts(x, ids, weights, w1, w2), want[0].detach().cpu(), rel, "out alone")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rest", [1, 17, 40, 129])
def test_blocks_that_end_early(mix, dtype, rest):
    """Every expert's last block holds a few rows, hidden ends inside a tile: waves without rows or
    columns leave the sums of the others alone."""
    experts, dim, hidden = 3, 520, 1304
    each = 256 * 12 + rest
    tokens = experts * each
    x, _, weights, w1, w2, dout = (t.cuda() for t in expert_inputs(dtype, tokens, experts, 1, dim,
                                                                   hidden, 62))
    ids = (torch.arange(tokens, dtype=torch.int32, device="cuda") % experts)[:, None].contiguous()
    want = experts_in_float64(x, ids, weights, w1, w2, dout)
    rel = expert_tolerance(dtype, dim, hidden, tokens)
    first = None
    for _ in range(3):
        out, saved = mix.experts_forward(x, ids, weights, w1, w2)
        got = (out, *mix.experts_backward(dout, x, ids, weights, w1, w2, saved))
        for g, v, name in zip(got, want, NAMES):
            near(g, v.detach().cpu(), rel, name)
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(got, first))


FAR = [(64, 904), (136, 904)]  # dim, hidden


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,hidden", FAR)
def test_tokens_beyond_32_bits(mix, dtype, dim, hidden):
    """Rows of x as rows of the first product, and as k of the gradient of w1."""
    x, ids, weights, w1, w2, dout = expert_inputs(dtype, 4300, 2, 2, dim, hidden, 64)
    a = [t.cuda() for t in (x, ids, weights, w1, w2)]
    out, saved = mix.experts_forward(*a)
    grads = mix.experts_backward(dout.cuda(), *a, saved)
    far = [far_apart(x), *a[1:]]
    far_out, far_saved = mix.experts_forward(*far)
    assert torch.equal(far_out, out)
    far_grads = mix.experts_backward(dout.cuda(), *far, far_saved)
    assert all(torch.equal(p, q) for p, q in zip(far_grads, grads))
