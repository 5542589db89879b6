"""Which derivatives of the mixture's operators there are: first ones by the backward pass, and an
error for all others (no GPU needed: the kernels are replaced by what fills their outputs)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_1503_08294_amd import gsn, mixture


@pytest.fixture(autouse=True)
def kernels(monkeypatch):
    """Every output is 1 (ids: 0)."""
    def fill(*outs):
        for t in outs:
            if t is not None:
                t.fill_(0 if t.dtype == torch.int32 else 1)

    monkeypatch.setattr(gsn, "gsn_layer_norm", lambda x, w, b, eps, y, stats=None: fill(y, stats))
    monkeypatch.setattr(gsn, "gsn_layer_norm_backward",
                        lambda dy, x, w, stats, dx, dw, db, ws: fill(dx, dw, db))
    monkeypatch.setattr(gsn, "gsn_route", lambda p, l, b, v, ids, w: fill(ids, w))
    monkeypatch.setattr(gsn, "gsn_route_backward", lambda p, dw, l, ids, dl: fill(dl))
    monkeypatch.setattr(gsn, "gsn_experts",
                        lambda p, x, ids, w, w1, w2, out, saved, ws: fill(out))
    monkeypatch.setattr(gsn, "gsn_experts_backward",
                        lambda p, dout, x, w, w1, w2, saved, dx, dw, dw1, dw2, ws:
                        fill(dx, dw, dw1, dw2))


IDS = torch.zeros(4, 2, dtype=torch.int32)
CALLS = {
    "layer_norm": (lambda x, w, b: mixture.layer_norm(x, w, b), [(4, 8), (8,), (8,)]),
    "route": (lambda l: mixture.route(l, 2)[1], [(4, 8)]),
    "experts": (lambda x, w, w1, w2: mixture.experts(x, IDS, w, w1, w2),
                [(4, 8), (4, 2), (3, 10, 8), (3, 8, 5)]),
}


@pytest.mark.parametrize("name", CALLS)
def test_first_derivatives(name):
    call, shapes = CALLS[name]
    a = [torch.ones(s, requires_grad=True) for s in shapes]
    call(*a).sum().backward()
    assert all(torch.equal(t.grad, torch.ones_like(t)) for t in a)


@pytest.mark.parametrize("name", CALLS)
def test_a_penalty_on_a_gradient_raises(name):
    call, shapes = CALLS[name]
    for i in range(len(shapes)):
        a = [torch.ones(s, requires_grad=True) for s in shapes]
        out = call(*a)
        grad, = torch.autograd.grad(out.sum(), a[i], create_graph=True)
        loss = out.sum() + grad.square().sum() + a[i].square().sum()
        with pytest.raises(RuntimeError, match="second time"):
            loss.backward()


@pytest.mark.parametrize("name", CALLS)
def test_a_recorded_backward_pass_that_is_not_differentiated(name):
    call, shapes = CALLS[name]
    a = [torch.ones(s, requires_grad=True) for s in shapes]
    grads = torch.autograd.grad(call(*a).sum(), a[:1], create_graph=True)
    assert torch.equal(grads[0], torch.ones_like(a[0]))
    a[0].square().sum().backward()
    assert torch.equal(a[0].grad, 2 * torch.ones_like(a[0]))


@pytest.mark.parametrize("name", CALLS)
def test_second_derivatives_through_the_gradient_that_comes_in(name):
    call, shapes = CALLS[name]
    a = [torch.ones(s) for s in shapes]
    a[0].requires_grad_()
    out = call(*a)
    v = torch.ones_like(out, requires_grad=True)
    grad, = torch.autograd.grad(out, a[0], v, create_graph=True)
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(grad.sum(), v)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("requires_grad", [False, True])
def test_a_tangent_is_refused(name, requires_grad):
    call, shapes = CALLS[name]
    for i in range(len(shapes)):
        a = [torch.ones(s, requires_grad=requires_grad) for s in shapes]
        with forward_ad.dual_level():
            call(*a)  # (no tangent: nothing to drop)
            a[i] = forward_ad.make_dual(a[i], torch.ones_like(a[i]))
            with pytest.raises(ValueError, match="tangent"):
                call(*a)
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                call(*a)
