"""What the mixture's C calls and their binding refuse on the host, before anything is enqueued
(no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1503_08294_amd import gsn, mixture

FAKE = 1 << 20  # never dereferenced: every call below fails validation first
INVAL, CAPACITY = gsn.GSN_E_INVAL, gsn.GSN_E_CAPACITY


def test_layer_norm_arguments():
    f = gsn._lib.gsn_layer_norm
    good = [gsn.GSN_BF16, gsn.GSN_F32, 4, 64, FAKE, 64, None, None, 1e-5, FAKE, 64, None, None]
    for at, bad in ((0, 3), (0, -1), (1, gsn.GSN_F16), (2, -1), (3, 0), (4, None), (5, 63),
                    (8, -1.0), (8, float("nan")), (9, None), (10, 63)):
        a = list(good)
        a[at] = bad
        assert f(*a) == INVAL, (at, bad)
    good[2] = 0
    assert f(*good) == gsn.GSN_OK  # no rows, nothing to do
    b = gsn._lib.gsn_layer_norm_backward
    ok = [gsn.GSN_F32, gsn.GSN_F32, 4, 64, FAKE, 64, FAKE, 64, None, FAKE, FAKE, 64, FAKE, FAKE,
          FAKE, 1 << 30, None]
    for at, bad, code in ((0, 7, INVAL), (2, -1, INVAL), (3, 0, INVAL), (4, None, INVAL),
                          (5, 1, INVAL), (6, None, INVAL), (7, 1, INVAL), (9, None, INVAL),
                          (11, 2, INVAL), (14, None, INVAL), (14, FAKE + 4, INVAL),
                          (15, 16, CAPACITY)):
        a = list(ok)
        a[at] = bad
        assert b(*a) == code, (at, bad)
    assert gsn.gsn_layer_norm_workspace_bytes(-1, 4) == 0
    assert gsn.gsn_layer_norm_workspace_bytes(4, 0) == 0
    assert gsn.gsn_layer_norm_workspace_bytes(0, 4) > 0


@pytest.mark.parametrize("bad", [dict(experts=0), dict(experts=1025), dict(top=0), dict(top=65),
                                 dict(top=9, experts=8), dict(score=2), dict(groups=0),
                                 dict(groups=5), dict(groups=65, experts=650),
                                 dict(top_groups=0), dict(top_groups=5), dict(best=0),
                                 dict(best=3), dict(top=5, top_groups=1),
                                 dict(scale=float("inf")), dict(scale=float("nan"))])
def test_route_parameters(bad):
    p = gsn.make_route(16, 2, groups=4, top_groups=2)
    for k, v in bad.items():
        setattr(p, k, v)
    assert gsn._lib.gsn_route(p, 0, 4, FAKE, 2000, None, None, FAKE, FAKE, None) == INVAL
    assert gsn._lib.gsn_route_backward(p, 0, 4, FAKE, FAKE, 2000, FAKE, FAKE, 2000,
                                       None) == INVAL


def test_route_arguments():
    p = gsn.make_route(16, 2)
    good = [p, 0, 4, FAKE, 16, None, None, FAKE, FAKE, None]
    for at, bad in ((0, None), (1, 3), (2, -1), (2, 1 << 40), (3, None), (4, 15), (7, None),
                    (8, None)):
        a = list(good)
        a[at] = bad
        assert gsn._lib.gsn_route(*a) == INVAL, (at, bad)
    good[2] = 0
    assert gsn._lib.gsn_route(*good) == gsn.GSN_OK
    good = [p, 0, 4, FAKE, FAKE, 16, FAKE, FAKE, 16, None]
    for at, bad in ((1, -1), (2, -1), (3, None), (4, None), (5, 3), (6, None), (7, None), (8, 3)):
        a = list(good)
        a[at] = bad
        assert gsn._lib.gsn_route_backward(*a) == INVAL, (at, bad)
    for a, code in (((-1, 4, FAKE, FAKE, None), INVAL), ((4, 0, FAKE, FAKE, None), INVAL),
                    ((4, 1025, FAKE, FAKE, None), INVAL), ((4, 4, None, FAKE, None), INVAL),
                    ((4, 4, FAKE, None, None), INVAL), ((1 << 31, 4, FAKE, FAKE, None), CAPACITY)):
        assert gsn._lib.gsn_route_counts(*a) == code
    for a in ((0, FAKE, 0.1, FAKE, None), (4, None, 0.1, FAKE, None), (4, FAKE, -0.1, FAKE, None),
              (4, FAKE, float("nan"), FAKE, None), (4, FAKE, 0.1, None, None)):
        assert gsn._lib.gsn_route_balance(*a) == INVAL


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(experts=0), dict(experts=1025), dict(top=0),
                                 dict(top=65), dict(dim=0), dict(dim=(1 << 20) + 1),
                                 dict(hidden=0), dict(hidden=(1 << 20) + 1), dict(tokens=-1),
                                 dict(tokens=(1 << 23) + 1), dict(tokens=1 << 22, top=32)])
def test_experts_parameters(bad):
    p = gsn.gsn_experts_params(gsn.GSN_BF16, 8, 2, 64, 32, 10)
    assert gsn.gsn_experts_workspace_bytes(p, False) > 0
    assert gsn.gsn_experts_saved_bytes(p) >= 4 * 10 * 2 * 2 * 32
    for k, v in bad.items():
        setattr(p, k, v)
    assert gsn.gsn_experts_workspace_bytes(p, False) == 0
    assert gsn.gsn_experts_workspace_bytes(p, True) == 0
    assert gsn.gsn_experts_saved_bytes(p) == 0
    assert gsn._lib.gsn_experts(p, FAKE, 1 << 21, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, FAKE,
                                1 << 40, None) == INVAL
    assert gsn._lib.gsn_experts_backward(p, FAKE, FAKE, 1 << 21, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                         FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == INVAL


def test_experts_arguments():
    p = gsn.gsn_experts_params(gsn.GSN_F32, 8, 2, 64, 32, 10)
    good = [p, FAKE, 64, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, FAKE, 1 << 30, None]
    for at, bad, code in ((1, None, INVAL), (2, 63, INVAL), (3, None, INVAL), (4, None, INVAL),
                          (5, None, INVAL), (6, None, INVAL), (7, None, INVAL),
                          (8, FAKE + 64, INVAL), (9, 100, CAPACITY), (10, None, INVAL),
                          (10, FAKE + 128, INVAL), (11, 100, CAPACITY)):
        a = list(good)
        a[at] = bad
        assert gsn._lib.gsn_experts(*a) == code, (at, bad)
    good = [p, FAKE, FAKE, 64, FAKE, FAKE, FAKE, FAKE, 1 << 30, FAKE, FAKE, FAKE, FAKE, FAKE,
            1 << 30, None]
    for at, bad, code in ((1, None, INVAL), (2, None, INVAL), (3, 1, INVAL), (4, None, INVAL),
                          (5, None, INVAL), (6, None, INVAL), (7, None, INVAL),
                          (7, FAKE + 8, INVAL), (8, 100, CAPACITY), (13, None, INVAL),
                          (13, FAKE + 8, INVAL), (14, 100, CAPACITY)):
        a = list(good)
        a[at] = bad
        assert gsn._lib.gsn_experts_backward(*a) == code, (at, bad)
    # more workgroups than a grid holds
    big = gsn.gsn_experts_params(gsn.GSN_F32, 1024, 1, 1 << 20, 1 << 20, 1)
    a = [big, FAKE, 1 << 20, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, FAKE, 1 << 40, None]
    assert gsn._lib.gsn_experts(*a) == CAPACITY


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device"):
        mixture.layer_norm(x)
    with pytest.raises(ValueError, match="2-dimensional"):
        mixture.layer_norm(torch.zeros(2, 4, 8))
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        mixture.layer_norm(x.double())
    with pytest.raises(ValueError, match="score"):
        mixture.route(x, 2, score="max")
    with pytest.raises(ValueError, match="device"):
        mixture.route(x, 2)
    ids, w = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    with pytest.raises(ValueError, match="3-dimensional"):
        mixture.experts(x, ids, w, torch.zeros(8, 8), torch.zeros(8, 8))
    with pytest.raises(ValueError, match="device"):
        mixture.experts(x, ids, w, torch.zeros(3, 8, 8), torch.zeros(3, 8, 4))
    with pytest.raises(gsn.GsnError):
        mixture.experts(x, ids[:, :0], w[:, :0], torch.zeros(3, 8, 8), torch.zeros(3, 8, 4))
    with pytest.raises(ValueError, match="device"):
        mixture.route_counts(ids, 4)
    assert ctypes.sizeof(gsn.gsn_route_params) == 32
    assert ctypes.sizeof(gsn.gsn_experts_params) == 32
