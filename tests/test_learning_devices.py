"""The learning calls on tensors of a device that is not the current one: the C call is made with
their device current and with that device's stream (no GPU needed: tensors, devices and the library
are stand-ins)."""
import pytest
import torch

from paper_1503_08294_amd import gsn, learning
from test_mixture_devices import OnDevice

F32, I32, U8, I8 = torch.float32, torch.int32, torch.uint8, torch.int8


def calls(d):
    """(name of the C call, the binding's call) with every tensor on device d."""
    def t(*shape, dtype=F32):
        return OnDevice(d, shape, dtype)

    ep = gsn.gsn_entropy_params(gsn.GSN_F32, 8, 20, 5)
    op = gsn.gsn_orthogonal_params(gsn.GSN_F32, 6, 8, 5, 3, *learning.COEFFICIENTS, 1e-7)
    lp = gsn.gsn_linear_params(gsn.GSN_F32, 8, 20, 5)
    x, w, m, ws = t(5, 8), t(20, 8), t(3, 6, 8), t(1 << 16, dtype=U8)
    return [
        ("gsn_cross_entropy", lambda: gsn.gsn_cross_entropy(
            ep, x, w, t(5, dtype=I32), t(20, dtype=U8), t(5), t(2, 5), ws)),
        ("gsn_cross_entropy_backward", lambda: gsn.gsn_cross_entropy_backward(
            ep, t(5), x, w, t(5, dtype=I32), t(20, dtype=U8), t(2, 5), x, w, ws)),
        ("gsn_orthogonalise", lambda: gsn.gsn_orthogonalise(op, m, m, ws)),
        ("gsn_orthogonal_step", lambda: gsn.gsn_orthogonal_step(
            op, m, m, m, 0.1, 0.9, 0.0, True, m, m, ws)),
        ("gsn_quantise", lambda: gsn.gsn_quantise(x, t(5, 8, dtype=I8), t(5))),
        ("gsn_linear_quantised", lambda: gsn.gsn_linear_quantised(
            lp, x, t(20, 8, dtype=I8), t(20), t(5, 20), ws)),
    ]


@pytest.mark.parametrize("device", [0, 1])
@pytest.mark.parametrize("at", range(6))
def test_the_tensors_device_is_current(monkeypatch, device, at):
    current, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append((name, current[0], args[-1]))
                return gsn.GSN_OK
            call.__name__ = name
            return call

    monkeypatch.setattr(gsn, "_current_device", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(gsn, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(gsn, "_lib", Library())
    name, call = calls(device)[at]
    call()
    assert seen == [(name, device, 1000 + device)]
    assert current == [0]


def test_tensors_of_two_devices_are_refused():
    x, far = OnDevice(0, (5, 8)), OnDevice(1, (20, 8))
    with pytest.raises(ValueError, match="not on"):
        learning.cross_entropy_forward(x, far, OnDevice(0, (5,), I32))
    with pytest.raises(ValueError, match="not on"):
        learning.cross_entropy_backward(OnDevice(1, (5,)), x, OnDevice(0, (20, 8)),
                                        OnDevice(0, (5,), I32), None, OnDevice(0, (2, 5)))
