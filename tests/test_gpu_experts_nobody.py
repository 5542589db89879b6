"""Batches of many tokens of which none has an expert, at sizes that take each of the products'
tiles."""
import pytest
import torch

from test_gpu_mixture import BF16, F16, F32, expert_inputs

pytestmark = pytest.mark.gpu


# (aligned sizes with 128 tiles of 256: sides of 256; others with 256 tiles of 128: sides of 128)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,experts,k,dim,hidden", [
    (3000, 4, 2, 1032, 1544), (3000, 4, 2, 515, 701), (300, 3, 1, 136, 72), (20, 64, 2, 72, 40)])
@pytest.mark.parametrize("foreign", [-1, 64, -(1 << 31), (1 << 31) - 1])
def test_nobody_has_an_expert(dtype, tokens, experts, k, dim, hidden, foreign):
    from paper_1503_08294_amd import mixture as mix
    a = [t.cuda() for t in expert_inputs(dtype, tokens, experts, k, dim, hidden, 63)]
    x, ids, weights, w1, w2, dout = a
    ids[:] = foreign
    x[:] = float("nan")  # nothing of it is read
    out, saved = mix.experts_forward(x, ids, weights, w1, w2)
    got = mix.experts_backward(dout, x, ids, weights, w1, w2, saved)
    assert not out.any() and not mix.experts(x, ids, weights, w1, w2).any()
    for g, like in zip(got, (x, weights, w1, w2)):
        assert g.shape == like.shape and not g.any()
