"""A training step recorded through autograd, and updates in place, replayed with the program's own
work between."""
import pytest
import torch

from paper_1503_08294_amd import learning

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tokens,classes,dim", [
    (torch.bfloat16, 70, 260, 48), (torch.float32, 300, 500, 33), (torch.float16, 20, 130, 64)])
def test_a_recorded_training_step(dtype, tokens, classes, dim):
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    def targets():
        return torch.randint(-1, classes, (tokens,), generator=g, device="cuda", dtype=torch.int32)

    cot = torch.rand(tokens, generator=g, device="cuda")
    # (other leaves than the recorded ones: no eager graph of theirs may live while they are recorded)
    v, u = randn(tokens, dim).requires_grad_(), randn(classes, dim).requires_grad_()
    torch.autograd.grad(learning.cross_entropy(v, u, targets()), (v, u), cot)
    torch.cuda.synchronize()
    x, w, t = randn(tokens, dim).requires_grad_(), randn(classes, dim).requires_grad_(), targets()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = learning.cross_entropy(x, w, t)
        dx, dw = torch.autograd.grad(loss, (x, w), cot)
    for _ in range(4):
        with torch.no_grad():
            x.copy_(randn(tokens, dim))
            w.copy_(randn(classes, dim))
            t.copy_(targets())
        graph.replay()
        torch.cuda.synchronize()
        y, z = x.detach(), w.detach()
        want, stats = learning.cross_entropy_forward(y, z, t)
        assert torch.equal(loss, want)
        for got, want in zip((dx, dw), learning.cross_entropy_backward(cot, y, z, t, None, stats)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,rows,cols", [(2, 40, 24), (3, 200, 312)])
def test_a_recorded_update_in_place(dtype, batch, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(2)
    w, d = (torch.randn(batch, rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    m = torch.randn(batch, rows, cols, generator=g, device="cuda")
    p, q = w.clone(), m.clone()
    learning.orthogonal_step(w, d, m, 0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        learning.orthogonal_step(w, d, m, 0.1, decay=0.1, out=(w, m))
    torch.cuda.synchronize()
    assert torch.equal(w, p) and torch.equal(m, q)  # (recorded, not run)
    for _ in range(4):
        d.copy_(torch.randn(batch, rows, cols, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        p, q = learning.orthogonal_step(p, d, q, 0.1, decay=0.1)
        assert torch.equal(w, p) and torch.equal(m, q)
