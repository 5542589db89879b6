"""The layer norm of the longest row that it takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_one_row_of_2_to_the_27():
    from paper_1503_08294_amd import mixture as mix
    dim = 1 << 27
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(1, dim, generator=g, device="cuda") for _ in range(2))
    w, b = (torch.randn(dim, generator=g, device="cuda") for _ in range(2))
    y, stats = mix.layer_norm_forward(x, w, b)
    got = (y, *mix.layer_norm_backward(dy, x, w, b, stats))
    xc = x.double() - x.double().mean()
    r = 1 / torch.sqrt(xc.square().mean() + 1e-5)
    n = xc * r
    gd = dy.double() * w.double()
    want = (n * w.double() + b.double(), r * (gd - gd.mean() - n * (gd * n).mean()),
            (dy.double() * n)[0], dy.double()[0])
    # sums of 2^19 terms a lane, whose errors grow as the root of their number, 8 for the safe side
    rel = 8 * (dim // 256) ** 0.5 * 2.0 ** -24
    for p, q, name in zip(got, want, ("y", "dx", "dweight", "dbias")):
        assert p.shape == q.shape and (p.double() - q).norm() <= rel * q.norm(), name
        assert (p.double() - q).abs().max() <= 16 * rel * q.abs().max(), name
