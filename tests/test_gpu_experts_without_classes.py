"""The example's training where a part of the model has no part in the loss."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("update", ["adam", "orthogonal"])
def test_classes_that_are_not_trained_stay(update):
    from paper_1503_08294_amd import local_experts
    g = torch.Generator().manual_seed(1)
    model = local_experts.LocalExperts(torch.randn(3, 8, generator=g).cuda(), 32, 24, classes=50)
    points = torch.randn(200, 3, generator=g).cuda()
    normals = torch.nn.functional.normalize(torch.randn(200, 3, generator=g), dim=1).cuda()
    before = {k: v.clone() for k, v in model.state_dict().items()}
    local_experts.train(model, points, normals, steps=2, batch=64, update=update)
    after = model.state_dict()
    assert torch.equal(after["classes"], before["classes"])
    assert not torch.equal(after["w1"], before["w1"])
    assert all(torch.isfinite(v).all() for v in after.values())
