"""Tensors that are not those that a call's parameters tell of: the kernels go by the parameters and
would read and write past the tensors' ends, so the binding refuses them before the library is called
(no GPU needed: tensors, devices and the library are stand-ins)."""
import pytest
import torch

from paper_1503_08294_amd import gsn, learning
from test_mixture_devices import OnDevice

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


def t(*shape, dtype=F32):
    return OnDevice(0, shape, dtype)


@pytest.fixture
def called(monkeypatch):
    """Names of the library's functions that were called."""
    names = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                names.append(name)
                return gsn.GSN_OK
            call.__name__ = name
            return call

    monkeypatch.setattr(gsn, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(gsn, "_raw_stream", lambda index: 1000)
    monkeypatch.setattr(gsn, "_lib", Library())
    return names


def matrices(rows=6, cols=8, batch=3, code=gsn.GSN_F32):
    return gsn.gsn_orthogonal_params(code, rows, cols, 5, batch, *learning.COEFFICIENTS, 1e-7)


ROOM = 1 << 16


@pytest.mark.parametrize("shape,fits", [
    ((3, 6, 8), True), ((1, 3, 6, 8), True), ((2, 6, 8), False), ((4, 6, 8), False),
    ((3, 8, 6), False), ((6, 8), False), ((3, 48), False), ((144,), False), ((3, 5, 8), False)])
def test_matrices_of_other_sizes(called, shape, fits):
    x = t(*shape)
    calls = [lambda: gsn.gsn_orthogonalise(matrices(), x, x, t(ROOM, dtype=U8)),
             lambda: gsn.gsn_orthogonal_step(matrices(), x, x, x, 0.1, 0.9, 0.0, True, x, x,
                                             t(ROOM, dtype=U8))]
    for call in calls:
        if fits:
            call()
        else:
            with pytest.raises(ValueError, match="must be 3 matrices of 6 x 8"):
                call()
    assert called == (["gsn_orthogonalise", "gsn_orthogonal_step"] if fits else [])


def test_one_matrix_by_itself(called):
    x = t(6, 8)
    gsn.gsn_orthogonalise(matrices(batch=1), x, x, t(ROOM, dtype=U8))
    assert called == ["gsn_orthogonalise"]


@pytest.mark.parametrize("code,fits", [(gsn.GSN_F32, False), (gsn.GSN_BF16, True),
                                       (gsn.GSN_F16, False), (7, False)])
def test_tensors_of_another_type(called, code, fits):
    """(An element of the parameters' type may be twice as long as the tensors'.)"""
    ep = gsn.gsn_entropy_params(code, 8, 20, 5)
    lp = gsn.gsn_linear_params(code, 8, 20, 5)
    xp = gsn.gsn_experts_params(code, 3, 2, 8, 4, 5)
    x, w, m, ws = t(5, 8, dtype=BF16), t(20, 8, dtype=BF16), t(3, 6, 8, dtype=BF16), t(ROOM, dtype=U8)
    targets, ids, pairs = t(5, dtype=torch.int32), t(5, 2, dtype=torch.int32), t(5, 2)
    w1, w2, f = t(3, 8, 8, dtype=BF16), t(3, 8, 4, dtype=BF16), t(3, 6, 8)
    calls = [
        lambda: gsn.gsn_cross_entropy(ep, x, w, targets, None, t(5), None, ws),
        lambda: gsn.gsn_cross_entropy_backward(ep, t(5), x, w, targets, None, t(2, 5), x, w, ws),
        lambda: gsn.gsn_orthogonalise(matrices(code=code), m, m, ws),
        lambda: gsn.gsn_orthogonal_step(matrices(code=code), m, m, f, 0.1, 0.9, 0.0, True, m, f, ws),
        lambda: gsn.gsn_linear_quantised(lp, x, t(20, 8, dtype=torch.int8), t(20),
                                         t(5, 20, dtype=BF16), ws),
        lambda: gsn.gsn_experts(xp, x, ids, pairs, w1, w2, x, ws, ws),
        lambda: gsn.gsn_experts_backward(xp, x, x, pairs, w1, w2, ws, x, pairs, w1, w2, ws)]
    for call in calls:
        if fits:
            call()
        else:
            with pytest.raises(ValueError, match="type that the parameters"):
                call()
    assert len(called) == (len(calls) if fits else 0)


def test_sizes_beyond_32_bits(monkeypatch):
    """They are out of every call's range, and not taken modulo 2^32 for one that is in it."""
    far = (1 << 32) + 8
    x = torch.zeros(1, 1)
    for call in (lambda: learning.orthogonalise(x, steps=(1 << 32) + 5),
                 lambda: learning.orthogonal_step(x, x, x, 0.1, steps=(1 << 32) + 5),
                 lambda: learning.orthogonalise(x, steps=-(1 << 32) + 5),
                 lambda: learning.cross_entropy(x.expand(1, far), x.expand(1, far), x),
                 lambda: learning.cross_entropy(x, x.expand(far, 1), x),
                 lambda: learning.linear_8bit(x.expand(1, far), x.expand(1, far), x)):
        with pytest.raises(gsn.GsnError):
            call()


def test_rows_beyond_32_bits(monkeypatch):
    seen = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append((name, args))
                return gsn.GSN_E_INVAL
            call.__name__ = name
            return call

    monkeypatch.setattr(gsn, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(gsn, "_raw_stream", lambda index: 1000)
    monkeypatch.setattr(gsn, "_lib", Library())
    far = (1 << 32) + 8
    x, s = t(2, far), t(2, 2)
    for call in (lambda: gsn.gsn_quantise(x, t(2, far, dtype=torch.int8), t(2)),
                 lambda: gsn.gsn_layer_norm(x, None, None, 1e-5, x),
                 lambda: gsn.gsn_layer_norm_backward(x, x, None, s, x, None, None, None)):
        with pytest.raises(gsn.GsnError):
            call()
    assert len(seen) == 3
    for name, args in seen:
        assert far not in args[:4] and -1 in args[:4], name
