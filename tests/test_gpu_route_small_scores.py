"""Scores far below the largest: their relative errors grow with the exponential's argument, as the
header says."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_error_of_small_scores(score):
    from paper_1503_08294_amd import mixture as mix
    g = torch.Generator().manual_seed(1)
    logits = -85 * torch.rand(300, 64, generator=g)
    logits[:, 5] = 0.0  # the largest
    ids, w = mix.route(logits.cuda(), 64, score=score, renormalise=False)
    l = logits.double().gather(1, ids.cpu().long())
    want = l.sigmoid() if score == "sigmoid" else \
        torch.exp(l) / logits.double().exp().sum(1, keepdim=True)
    error = (w.double().cpu() - want).abs() / want
    # the product with log2 e is rounded, and log2 e itself by 0.22 of 2^-24: 1.25 |v|; a unit or
    # two of the power of two, of the sum of up to 64 terms (one of 1, the others decaying) and of
    # its reciprocal or quotient: 16
    assert (error <= (1.25 * l.abs() + 16) * 2.0 ** -24).all(), (error * 2 ** 24).max().item()
    near_zero = error[l > -4].max().item() * 2 ** 24
    far = error[l < -60].max().item() * 2 ** 24
    assert far > near_zero  # (what the growth is)
