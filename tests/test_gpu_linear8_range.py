"""Layers in 8 bits where a row's scale and a column's are far from 1, one large and one small: the
result is a number though the sum times one of them is not."""
import pytest
import torch

import learning_reference as ref
from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,dim,out", [(1, 100, 33), (2, 64, 64), (5, 200, 70), (70, 100, 64),
                                            (70, 64, 33), (300, 256, 400), (1_100, 130, 520)])
@pytest.mark.parametrize("x_size,w_size", [(1e37, 1e-30), (1e-30, 1e37), (1e37, 1e-38),
                                           (1e-37, 1e30), (1e37, 1.0)])
def test_scales_far_from_one(dtype, tokens, dim, out, x_size, w_size):
    g = torch.Generator().manual_seed(tokens + out)
    x = (torch.randn(tokens, dim, generator=g).clamp(-3, 3) * x_size).to(dtype)
    w = torch.randint(-127, 128, (out, dim), generator=g).to(torch.int8)
    w[0] = 0
    scales = (torch.rand(out, generator=g) + 0.5) / 127 / dim * w_size
    want, tol = ref.linear_8bit(x, w, scales)
    got = learning.linear_8bit(x.cuda(), w.cuda(), scales.cuda()).double().cpu()
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol).all()
