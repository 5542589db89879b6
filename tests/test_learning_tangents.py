"""Forward-mode tangents that the halves of the cross entropy would drop (no GPU needed)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_1503_08294_amd import learning


@pytest.mark.parametrize("at", range(2))
def test_the_forward_half_refuses_them(at):
    args = [torch.zeros(4, 8), torch.zeros(5, 8)]
    with forward_ad.dual_level():
        args[at] = forward_ad.make_dual(args[at], torch.ones_like(args[at]))
        with pytest.raises(ValueError, match="forward-mode tangent"):
            learning.cross_entropy_forward(*args, torch.zeros(4, dtype=torch.int32))


@pytest.mark.parametrize("at", [0, 1, 2, 5])
def test_the_backward_half_refuses_them(at):
    """(Of the gradient that comes in too: a derivative of the backward pass, forward over reverse.)"""
    args = [torch.zeros(4), torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32),
            None, torch.zeros(2, 4)]
    with forward_ad.dual_level():
        args[at] = forward_ad.make_dual(args[at], torch.ones_like(args[at]))
        with pytest.raises(ValueError, match="forward-mode tangent"):
            learning.cross_entropy_backward(*args)
