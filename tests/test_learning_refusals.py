"""What the calls that train and serve a model over the units refuse on the host, before anything is
enqueued (no GPU needed)."""
import pytest
import torch

from paper_1503_08294_amd import gsn, learning

FAKE = 1 << 20  # never dereferenced: every call below fails validation first
OK, INVAL, CAPACITY = gsn.GSN_OK, gsn.GSN_E_INVAL, gsn.GSN_E_CAPACITY
LOTS = 1 << 60


def each(f, good, cases):
    for at, bad, code in cases:
        a = list(good)
        a[at] = bad
        assert f(*a) == code, (at, bad)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(dim=0), dict(dim=65_537),
                                 dict(classes=0), dict(classes=(1 << 28) + 1), dict(tokens=-1),
                                 dict(tokens=(1 << 24) + 1)])
def test_entropy_parameters(bad):
    p = gsn.gsn_entropy_params(gsn.GSN_BF16, 64, 100, 8)
    assert gsn.gsn_cross_entropy_workspace_bytes(p, False) > 0
    assert gsn.gsn_cross_entropy_workspace_bytes(p, True) > 0
    for k, v in bad.items():
        setattr(p, k, v)
    assert gsn.gsn_cross_entropy_workspace_bytes(p, False) == 0
    assert gsn._lib.gsn_cross_entropy(p, FAKE, 1 << 17, FAKE, 1 << 17, FAKE, None, FAKE, None, FAKE,
                                      LOTS, None) == INVAL
    assert gsn._lib.gsn_cross_entropy_backward(p, FAKE, FAKE, 1 << 17, FAKE, 1 << 17, FAKE, None,
                                               FAKE, FAKE, FAKE, FAKE, LOTS, None) == INVAL


def test_entropy_arguments():
    p = gsn.gsn_entropy_params(gsn.GSN_F32, 64, 100, 8)
    good = [p, FAKE, 64, FAKE, 64, FAKE, None, FAKE, None, FAKE, LOTS, None]
    each(gsn._lib.gsn_cross_entropy, good,
         [(0, None, INVAL), (1, None, INVAL), (2, 63, INVAL), (3, None, INVAL), (4, 63, INVAL),
          (5, None, INVAL), (7, None, INVAL), (9, None, INVAL), (9, FAKE + 16, INVAL),
          (10, gsn.gsn_cross_entropy_workspace_bytes(p, False) - 1, CAPACITY)])
    back = [p, FAKE, FAKE, 64, FAKE, 64, FAKE, None, FAKE, FAKE, FAKE, FAKE, LOTS, None]
    each(gsn._lib.gsn_cross_entropy_backward, back,
         [(0, None, INVAL), (1, None, INVAL), (2, None, INVAL), (3, 1, INVAL), (4, None, INVAL),
          (5, 63, INVAL), (6, None, INVAL), (8, None, INVAL), (11, None, INVAL),
          (11, FAKE + 8, INVAL),
          (12, gsn.gsn_cross_entropy_workspace_bytes(p, True) - 1, CAPACITY)])
    back[9] = back[10] = None
    assert gsn._lib.gsn_cross_entropy_backward(*back) == OK  # nothing wanted
    p.tokens = 0
    assert gsn._lib.gsn_cross_entropy(*good) == OK
    # more tiles than a grid takes
    p = gsn.gsn_entropy_params(gsn.GSN_BF16, 1 << 16, 1 << 20, 1 << 24)
    back[0], back[3], back[5], back[9], back[10] = p, 1 << 16, 1 << 16, FAKE, FAKE
    assert gsn._lib.gsn_cross_entropy_backward(*back) == CAPACITY


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(rows=0), dict(cols=0), dict(rows=32_769), dict(cols=32_769),
    dict(steps=0), dict(steps=65), dict(batch=-1), dict(batch=(1 << 20) + 1), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(a=float("nan")), dict(a=6.0),
    dict(b=5.0), dict(c=-30.0), dict(a=29.0, b=-29.0)])
def test_orthogonal_parameters(bad):
    p = gsn.gsn_orthogonal_params(gsn.GSN_F32, 8, 9, 5, 2, *learning.COEFFICIENTS, 1e-7)
    assert gsn.gsn_orthogonal_workspace_bytes(p, False) > 0
    for k, v in bad.items():
        setattr(p, k, v)
    assert gsn.gsn_orthogonal_workspace_bytes(p, True) == 0
    assert gsn._lib.gsn_orthogonalise(p, FAKE, FAKE, FAKE, LOTS, None) == INVAL
    assert gsn._lib.gsn_orthogonal_step(p, FAKE, FAKE, FAKE, 0.1, 0.9, 0.0, 1, FAKE, FAKE, FAKE,
                                        LOTS, None) == INVAL


def test_orthogonal_arguments():
    p = gsn.gsn_orthogonal_params(gsn.GSN_F16, 8, 9, 5, 2, *learning.COEFFICIENTS, 1e-7)
    size = gsn.gsn_orthogonal_workspace_bytes
    each(gsn._lib.gsn_orthogonalise, [p, FAKE, FAKE, FAKE, LOTS, None],
         [(0, None, INVAL), (1, None, INVAL), (2, None, INVAL), (3, None, INVAL),
          (3, FAKE + 128, INVAL), (4, size(p, False) - 1, CAPACITY)])
    w, g, m, new_w, new_m = (FAKE * i for i in range(1, 6))
    good = [p, w, g, m, 0.1, 0.9, 0.0, 1, new_w, new_m, FAKE, LOTS, None]
    nan = float("nan")
    # outputs over what is still read: not the weights or the gradient for the momentum, nor either
    # momentum for the weights
    each(gsn._lib.gsn_orthogonal_step, good,
         [(9, g, INVAL), (9, w, INVAL), (9, new_w, INVAL), (8, m, INVAL)])
    each(gsn._lib.gsn_orthogonal_step, good,
         [(0, None, INVAL), (1, None, INVAL), (2, None, INVAL), (3, None, INVAL), (4, nan, INVAL),
          (5, nan, INVAL), (6, float("inf"), INVAL), (8, None, INVAL), (9, None, INVAL),
          (10, None, INVAL), (10, FAKE + 1, INVAL), (11, size(p, True) - 1, CAPACITY)])
    p.batch = 0
    assert gsn._lib.gsn_orthogonalise(p, None, None, None, 0, None) == OK
    p = gsn.gsn_orthogonal_params(gsn.GSN_F16, 1 << 15, 1 << 15, 5, 1 << 10,
                                  *learning.COEFFICIENTS, 1e-7)
    assert gsn._lib.gsn_orthogonalise(p, FAKE, FAKE, FAKE, LOTS, None) == CAPACITY


def test_quantise_arguments():
    each(gsn._lib.gsn_quantise, [gsn.GSN_BF16, 4, 64, FAKE, 64, FAKE, 64, FAKE, None],
         [(0, 3, INVAL), (0, -1, INVAL), (1, -1, INVAL), (2, 0, INVAL), (2, (1 << 27) + 1, INVAL),
          (3, None, INVAL), (4, 63, INVAL), (5, None, INVAL), (6, 63, INVAL), (7, None, INVAL),
          (1, 0, OK)])


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dim=0), dict(dim=1 << 17), dict(out=0),
                                 dict(out=(1 << 28) + 1), dict(tokens=-1),
                                 dict(tokens=(1 << 24) + 1)])
def test_linear_parameters(bad):
    p = gsn.gsn_linear_params(gsn.GSN_BF16, 64, 100, 8)
    assert gsn.gsn_linear_quantised_workspace_bytes(p) > 0
    for k, v in bad.items():
        setattr(p, k, v)
    assert gsn.gsn_linear_quantised_workspace_bytes(p) == 0
    assert gsn._lib.gsn_linear_quantised(p, FAKE, 1 << 18, FAKE, 1 << 18, FAKE, FAKE, 1 << 30,
                                         FAKE, LOTS, None) == INVAL


def test_linear_arguments():
    p = gsn.gsn_linear_params(gsn.GSN_BF16, 64, 100, 8)
    each(gsn._lib.gsn_linear_quantised, [p, FAKE, 64, FAKE, 64, FAKE, FAKE, 100, FAKE, LOTS, None],
         [(0, None, INVAL), (1, None, INVAL), (2, 63, INVAL), (3, None, INVAL), (4, 63, INVAL),
          (5, None, INVAL), (6, None, INVAL), (7, 99, INVAL), (8, None, INVAL),
          (8, FAKE + 64, INVAL),
          (9, gsn.gsn_linear_quantised_workspace_bytes(p) - 1, CAPACITY)])
    p.tokens, p.out = 1 << 24, 1 << 16
    assert gsn._lib.gsn_linear_quantised(p, FAKE, 64, FAKE, 64, FAKE, FAKE, 1 << 16, FAKE, LOTS,
                                         None) == CAPACITY


def test_tensors_of_the_host_are_refused():
    x, w = torch.zeros(4, 8), torch.zeros(5, 8)
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        learning.cross_entropy(x, w, t)
    with pytest.raises(ValueError, match="device tensor"):
        learning.orthogonalise(x)
    with pytest.raises(ValueError, match="device tensor"):
        learning.orthogonal_step(x, x, x, 0.1)
    with pytest.raises(ValueError, match="device tensor"):
        learning.quantise(x)
    with pytest.raises(ValueError, match="device tensor"):
        learning.linear_8bit(x, w.to(torch.int8), torch.zeros(5))


def test_shapes_are_refused():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="2-dimensional"):
        learning.cross_entropy(x[0], x, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="2-dimensional"):
        learning.cross_entropy(x, x[0], torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="a matrix or a batch"):
        learning.orthogonalise(x[0])
    with pytest.raises(ValueError, match="2-dimensional"):
        learning.quantise(x[0])
    with pytest.raises(ValueError, match="2-dimensional"):
        learning.linear_8bit(x, x[0].to(torch.int8), x[0])
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        learning.orthogonalise(x.double())


def test_a_gradient_that_there_is_none_of_is_refused():
    x = torch.zeros(4, 8, requires_grad=True)
    for f in (lambda: learning.orthogonalise(x), lambda: learning.quantise(x),
              lambda: learning.orthogonal_step(x, x, x, 0.1),
              lambda: learning.linear_8bit(x, x, x)):
        with pytest.raises(ValueError, match="no derivative"):
            f()
    with torch.no_grad(), pytest.raises(ValueError, match="device tensor"):
        learning.orthogonalise(x)


def test_a_tangent_is_refused():
    import torch.autograd.forward_ad as fwd
    x = torch.zeros(4, 8)
    with fwd.dual_level():
        d = fwd.make_dual(x, torch.ones_like(x))
        for f in (lambda: learning.cross_entropy(d, x, None), lambda: learning.orthogonalise(d),
                  lambda: learning.quantise(d), lambda: learning.linear_8bit(d, x, x),
                  lambda: learning.orthogonal_step(x, d, x, 0.1)):
            with pytest.raises(ValueError, match="forward-mode tangent"):
                f()
