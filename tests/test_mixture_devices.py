"""The mixture's calls on tensors of a device that is not the current one: the C call is made with
their device current and with that device's stream (no GPU needed: tensors, devices and the library
are stand-ins)."""
from types import SimpleNamespace

import pytest
import torch

from paper_1503_08294_amd import gsn, mixture

F32, I32, U8 = torch.float32, torch.int32, torch.uint8


class OnDevice:
    """As much of a contiguous device tensor as the binding looks at."""
    is_cuda = True

    def __init__(self, index, shape, dtype=F32):
        self.device, self.shape, self.dtype = SimpleNamespace(index=index), shape, dtype

    def get_device(self):
        return self.device.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self):
        return (self.shape[-1], 1)

    def data_ptr(self):
        return 1 << 20

    def is_contiguous(self):
        return True


def calls(d):
    """(name of the C call, the binding's call) with every tensor on device d."""
    def t(*shape, dtype=F32):
        return OnDevice(d, shape, dtype)

    p = gsn.make_route(8, 2)
    ep = gsn.gsn_experts_params(gsn.GSN_F32, 3, 2, 8, 4, 5)
    x, ids, w, w1, w2 = t(5, 8), t(5, 2, dtype=I32), t(5, 2), t(3, 8, 8), t(3, 8, 4)
    ws = t(1 << 16, dtype=U8)
    return [
        ("gsn_layer_norm", lambda: gsn.gsn_layer_norm(x, t(8), t(8), 1e-5, x, t(2, 5))),
        ("gsn_layer_norm_backward", lambda: gsn.gsn_layer_norm_backward(
            x, x, t(8), t(2, 5), x, t(8), t(8), ws)),
        ("gsn_route", lambda: gsn.gsn_route(p, x, t(8), t(5, dtype=U8), ids, w)),
        ("gsn_route_backward", lambda: gsn.gsn_route_backward(p, w, x, ids, x)),
        ("gsn_route_counts", lambda: gsn.gsn_route_counts(ids, t(8, dtype=I32))),
        ("gsn_route_balance", lambda: gsn.gsn_route_balance(t(8, dtype=I32), 0.1, t(8))),
        ("gsn_experts", lambda: gsn.gsn_experts(ep, x, ids, w, w1, w2, x, ws, ws)),
        ("gsn_experts_backward", lambda: gsn.gsn_experts_backward(
            ep, x, x, w, w1, w2, ws, x, w, w1, w2, ws)),
    ]


@pytest.mark.parametrize("device", [0, 1])
@pytest.mark.parametrize("at", range(8))
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


def test_counts_and_balance_are_on_one_device():
    counts, balance = OnDevice(0, (8,), I32), OnDevice(1, (8,))
    with pytest.raises(ValueError, match="not on"):
        mixture.route_balance(counts, balance)
