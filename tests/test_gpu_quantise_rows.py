"""Rows in 8 bits where there are many of them: a wave's or a workgroup's, of any length and stride,
with rows among them that are not finite, and what lies beside them."""
from __future__ import annotations

import pytest
import torch

import learning_reference as ref
from paper_1503_08294_amd import gsn, learning

pytestmark = pytest.mark.gpu

TYPES = (torch.float32, torch.bfloat16, torch.float16)


def _rows(rows, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, dim, generator=g) * torch.logspace(-3, 3, rows)[:, None]
    x[5] = torch.inf
    x[rows // 2, dim // 2] = torch.nan
    x[rows - 2] = 0.0
    if dim > 2:
        x[7] = torch.randint(-254, 255, (dim,), generator=g) / 2  # ties
        x[7, 1] = 127.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(2049, 1), (2048, 7), (2050, 8), (2051, 65), (4099, 515),
                                      (2048, 1024), (2047, 1024), (2303, 1025), (4096, 2048),
                                      (4095, 2047), (4111, 2049), (2077, 2500), (66000, 9)])
def test_many_rows(dtype, rows, dim):
    x = _rows(rows, dim, dtype, rows + dim)
    want_q, want_s = ref.quantise(x)
    q, s = learning.quantise(x.cuda())
    assert torch.equal(s.cpu().nan_to_num(-1), want_s.nan_to_num(-1))
    assert torch.equal(q.cpu().long(), want_q)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(2051, 65), (2049, 1001), (33, 1003), (3, 17001)])
def test_rows_of_wider_tensors(dtype, rows, dim):
    """Rows that start at any element, of x and of q; what is beside q's rows stays."""
    x = _rows(rows, dim, dtype, dim) if rows > 9 else torch.randn(
        rows, dim, generator=torch.Generator().manual_seed(dim)).to(dtype)
    want_q, want_s = ref.quantise(x)
    wide = torch.full((rows, dim + 6), torch.nan, dtype=dtype, device="cuda")
    wide[:, 3:3 + dim] = x.cuda()
    q = torch.full((rows, dim + 9), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    gsn.gsn_quantise(wide[:, 3:3 + dim], q[:, 5:5 + dim], s)
    torch.cuda.synchronize()
    assert torch.equal(s.cpu().nan_to_num(-1), want_s.nan_to_num(-1))
    assert torch.equal(q[:, 5:5 + dim].cpu().long(), want_q)
    assert (q[:, :5] == 99).all() and (q[:, 5 + dim:] == 99).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,dim,out", [(2049, 1001, 70), (2051, 64, 33), (4100, 2040, 129),
                                            (2, 16381, 40), (2, 16390, 40)])
def test_layers_of_many_tokens(dtype, tokens, dim, out):
    g = torch.Generator().manual_seed(tokens + out)
    x = torch.randn(tokens, dim, generator=g).to(dtype)
    w, scales = learning.quantise((torch.randn(out, dim, generator=g) * dim ** -0.5).cuda())
    want, tol = ref.linear_8bit(x, w.cpu(), scales.cpu())
    got = learning.linear_8bit(x.cuda(), w, scales).double().cpu()
    assert ((got - want).abs() <= tol).all()
