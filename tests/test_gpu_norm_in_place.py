"""The layer norm's backward pass where dx is the memory of dy or of x: the sums over the rows are
those of what was there, whatever order dx is written in."""
import pytest
import torch

import mixture_reference as ref
from test_gpu_mixture import BF16, F16, F32, TYPES, close, randn

pytestmark = pytest.mark.gpu


def check_in_place(dtype, rows, dim, pad, wanted, over="dy"):
    from paper_1503_08294_amd import gsn, mixture
    x = randn(rows, dim, seed=1, dtype=dtype, scale=2.0) + 0.5
    w = 1 + 0.2 * randn(dim, seed=2)
    dy = randn(rows, dim, seed=4, dtype=dtype)
    _, stats = mixture.layer_norm_forward(x.cuda(), w.cuda(), None, 1e-5)
    _, want, dw, db = ref.layer_norm(x, w, None, 1e-5, dy)
    wide = torch.full((rows, dim + pad), 7.0, dtype=dtype, device="cuda")
    both = wide[:, :dim]
    both.copy_(dy if over == "dy" else x)
    dweight, dbias = (torch.empty(dim, device="cuda") if n in wanted else None
                      for n in ("dweight", "dbias"))
    ws = torch.empty(gsn.gsn_layer_norm_workspace_bytes(rows, dim), dtype=torch.uint8,
                     device="cuda")
    a = (both, x.cuda()) if over == "dy" else (dy.cuda(), both)
    gsn.gsn_layer_norm_backward(*a, w.cuda(), stats, both, dweight, dbias, ws)
    # one rounding of dx; binary32 sums of D terms, D / 64 at a time by a lane and joined in a few
    # steps, in the mean, in r and in the two means of the gradient; over the rows, sums of as many
    # terms.  An error of f mean|x| in the mean shifts every n by r times that.
    r = 1 / torch.sqrt(x.double().var(1, correction=0, keepdim=True) + 1e-5)
    n = (x.double() - x.double().mean(1, keepdim=True)) * r
    g = dy.double().abs() * w.double().abs()
    size = r * (g + g.mean(1, keepdim=True) + n.abs() * (g * n.abs()).mean(1, keepdim=True))
    f = (dim / 64 + 24) * 2.0 ** -24
    shift = f * x.double().abs().mean(1, keepdim=True) * r
    close(both, want, ref.HALF_ULP[dtype] * want.abs() + f * size + shift * 3 * size
          + 2.0 ** -25 * (dtype == F16), "dx")
    assert (wide[:, dim:] == 7.0).all()
    f = (rows + 16) * 2.0 ** -24
    if dweight is not None:
        ny = (dy.double().abs() * (n.abs() * (f + (dim / 64 + 16) * 2.0 ** -24) + shift)).sum(0)
        close(dweight, dw, 2.0 ** -24 * dw.abs() + ny, "dweight")
    if dbias is not None:
        close(dbias, db, 2.0 ** -24 * db.abs() + f * dy.double().abs().sum(0), "dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(1, 64), (27, 704), (512, 300), (512, 2048), (513, 300),
                                      (300, 4100), (3, 20_003), (600, 9000)])
def test_dx_over_dy(dtype, rows, dim):
    """Few rows (sums beside the rows' workgroups where dx lies apart), more of them, and rows that
    are longer than a workgroup's registers hold."""
    check_in_place(dtype, rows, dim, 0, ("dweight", "dbias"))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(27, 704), (5, 20_003)])
@pytest.mark.parametrize("wanted", [("dweight",), ("dbias",), ()])
def test_dx_over_dy_in_rows_of_a_wider_tensor(dtype, rows, dim, wanted):
    check_in_place(dtype, rows, dim, 9, wanted)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad", [(1, 64, 0), (27, 704, 0), (512, 2048, 0), (513, 300, 0),
                                          (27, 704, 9), (3, 20_003, 0), (300, 9000, 9)])
def test_dx_over_x(dtype, rows, dim, pad):
    check_in_place(dtype, rows, dim, pad, ("dweight", "dbias"), over="x")
