"""Weights whose gradients would be more tiles than a grid holds: what does without these runs."""
import pytest
import torch

from test_gpu_mixture import expert_tolerance, near

pytestmark = pytest.mark.gpu


def test_only_the_launches_of_a_call_count():
    from paper_1503_08294_amd import gsn, mixture as mix
    experts, hidden, dtype = 1024, 1 << 20, torch.bfloat16
    w1 = torch.zeros(experts, 2 * hidden, 1, dtype=dtype, device="cuda")
    w2 = torch.zeros(experts, 1, hidden, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    w1[-1] = torch.randn(2 * hidden, 1, generator=g, device="cuda").to(dtype)
    w2[-1] = (torch.randn(1, hidden, generator=g, device="cuda") / hidden ** 0.5).to(dtype)
    x = torch.tensor([[0.75]], dtype=dtype, device="cuda")
    dout = torch.tensor([[1.25]], dtype=dtype, device="cuda")
    ids = torch.tensor([[experts - 1]], dtype=torch.int32, device="cuda")
    weights = torch.tensor([[0.5]], device="cuda")
    xd, wd = x.double().requires_grad_(), weights.double().requires_grad_()
    h = (w1[-1].double() @ xd[0])
    want = (w2[-1].double() @ (torch.nn.functional.silu(h[:hidden]) * h[hidden:]))[None] * wd
    dx, dweights = torch.autograd.grad(want, (xd, wd), dout.double())
    rel = expert_tolerance(dtype, 1, hidden, 1)
    near(mix.experts(x, ids, weights, w1, w2), want.detach().cpu(), rel, "out alone")
    out, saved = mix.experts_forward(x, ids, weights, w1, w2)
    near(out, want.detach().cpu(), rel, "out")
    need = (True, True, False, False)
    got = mix.experts_backward(dout, x, ids, weights, w1, w2, saved, need)
    near(got[0], dx.cpu(), rel, "dx")
    near(got[1], dweights.cpu(), rel, "dweights")
    with pytest.raises(gsn.GsnError) as e:
        mix.experts_backward(dout, x, ids, weights, w1, w2, saved, (False, False, True, False))
    assert e.value.code == gsn.GSN_E_CAPACITY
