"""An update in place is one for autograd too: what was computed from the tensors before cannot be
differentiated through them afterwards (no GPU needed: the C call is a stand-in)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_1503_08294_amd import gsn, learning


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(gsn, "gsn_orthogonal_step", lambda *a: made.append(a))
    return made


def step(w, m, out, rate=0.1):
    with torch.no_grad():
        return learning.orthogonal_step(w, torch.ones_like(w), m, rate, out=out)


def test_a_graph_that_saved_the_weights_raises(calls):
    w, m = torch.ones(3, 4, requires_grad=True), torch.zeros(3, 4)
    loss = (w * w).sum()
    step(w, m, (w, m))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    (w * w).sum().backward()  # a graph of the new weights
    assert len(calls) == 1


def test_both_outputs_count_as_written(calls):
    w, m, p, q = (torch.ones(3, 4) for _ in range(4))
    before = [t._version for t in (w, m, p, q)]
    step(w, m, (p, q))
    assert [t._version - b for t, b in zip((w, m, p, q), before)] == [0, 0, 1, 1]
    assert step(w, m, None)[0] is not w and w._version == before[0]


def test_tensors_of_inference_mode(calls):
    with torch.inference_mode():
        w, m = torch.ones(3, 4), torch.zeros(3, 4)
        step(w, m, (w, m))
    v, n = torch.ones(3, 4), torch.zeros(3, 4)
    with torch.inference_mode():
        step(v, n, (v, n))
    assert len(calls) == 2


def test_outputs_that_want_a_derivative_are_refused(calls):
    w, m = torch.ones(3, 4), torch.zeros(3, 4)
    p = torch.ones(3, 4, requires_grad=True)
    with pytest.raises(ValueError, match="no derivative"):
        learning.orthogonal_step(w, w, m, 0.1, out=(p, m))
    with forward_ad.dual_level():
        d = forward_ad.make_dual(torch.zeros(3, 4), torch.ones(3, 4))
        with pytest.raises(ValueError, match="forward-mode tangent"):
            learning.orthogonal_step(w, w, m, 0.1, out=(w, d))
    assert not calls
