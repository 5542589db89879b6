"""A grown network as the gate of local models: ``python -m paper_1503_08294_amd.local_experts``.

A network is grown on a genus-3 surface; each of its units becomes an expert.  For a point, the
scores of the experts are the negative squared distances to the units (plus a term that is
learned), the two best answer, and what they say is added to the point's features: a layer norm,
``mixture.route``, ``mixture.experts``.  The model learns the surface's normals by the backward
passes of the three, the pairs an expert are evened out by ``mixture.route_counts`` and
``mixture.route_balance``, and single points are answered afterwards.

With ``--classes N`` it learns besides which of a second network's N units is nearest to a point, by
``learning.cross_entropy`` over the units, and names it with the units' weights in 8 bits
(``learning.quantise``, ``learning.linear_8bit``).  With ``--update orthogonal`` the experts' weights
and the units' are updated by ``learning.orthogonal_step``, the rest by Adam.
"""
from __future__ import annotations

import argparse
import json

import numpy as np
import torch

from . import clouds, gsn, learning, mixture


def grow_units(cloud: np.ndarray, units: int, seed: int = 1) -> torch.Tensor:
    """(3, units) float32 positions of a network grown on the cloud (n, 3) on the GPU."""
    soa = torch.from_numpy(np.ascontiguousarray(cloud.T)).cuda()
    net = gsn.Network(gsn.make_params(eps_n=0.006, n_max=units, e_max=4 * units + 16, m_max=16),
                      soa[:, :2].contiguous())
    net.run_schedule(soa, gsn.make_schedule(m_cap=16, insert_every=50,
                                            max_signals=2_048 * units, seed=seed))
    xyz = net.export()["xyz"].cuda()
    net.close()
    return xyz.contiguous()


def nearest_units(units: torch.Tensor, points: torch.Tensor) -> torch.Tensor:
    """(n,) int32: the unit of (3, units) that is nearest to each of the points (n, 3)."""
    n, count = units.shape[1], points.shape[0]
    net = gsn.Network(gsn.make_params(n_max=n, e_max=4 * n + 16, m_max=count), units)
    winners = net.find_winners(points.t().contiguous())[0].clone()
    net.close()
    return winners


def genus3_normals(points: np.ndarray) -> np.ndarray:
    """Unit gradients (n, 3) of the distance to the surface's skeleton, by differences."""
    h = 1e-5
    grad = np.stack([clouds.genus3_distance(points + h * a) - clouds.genus3_distance(points - h * a)
                     for a in np.eye(3)], axis=1)
    return (grad / np.linalg.norm(grad, axis=1, keepdims=True)).astype(np.float32)


class LocalExperts(torch.nn.Module):
    """points (n, 3) float32 -> normals (n, 3): waves of the point as features, one layer of
    local experts over them, and a linear answer.  The experts compute in ``dtype``; their
    weights are kept in float32 and rounded for each pass."""

    def __init__(self, units: torch.Tensor, dim=64, hidden=64, top=2, dtype=torch.bfloat16,
                 seed=0, classes=0):
        super().__init__()
        experts, device = units.shape[1], units.device
        g = torch.Generator().manual_seed(seed)

        def randn(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(device)

        self.top, self.dtype = top, dtype
        self.register_buffer("units", units.t().contiguous())
        self.register_buffer("waves", randn(3, dim // 2, scale=2.0))
        self.register_buffer("balance", torch.zeros(experts, device=device))
        spread = torch.cdist(self.units, self.units).topk(2, largest=False).values[:, 1].mean()
        self.sharpness = torch.nn.Parameter(1 / spread ** 2)
        self.router = torch.nn.Parameter(randn(dim, experts, scale=0.01))
        self.norm_weight = torch.nn.Parameter(torch.ones(dim, device=device))
        self.norm_bias = torch.nn.Parameter(torch.zeros(dim, device=device))
        self.w1 = torch.nn.Parameter(randn(experts, 2 * hidden, dim, scale=dim ** -0.5))
        self.w2 = torch.nn.Parameter(randn(experts, dim, hidden, scale=hidden ** -0.5))
        self.answer = torch.nn.Parameter(randn(dim, 3, scale=dim ** -0.5))
        # weights of the classes that features are told apart by, if there are any
        self.classes = torch.nn.Parameter(randn(classes, dim, scale=dim ** -0.5)) if classes \
            else None

    def features(self, points):
        """(features (n, dim), ids): ids (n, top) are the experts that answered, best first."""
        angle = points @ self.waves
        h = torch.cat([angle.sin(), angle.cos()], 1)
        y = mixture.layer_norm(h.to(self.dtype), self.norm_weight, self.norm_bias)
        d2 = (points[:, None] - self.units).square().sum(2)
        logits = y.float() @ self.router - self.sharpness * d2
        ids, weights = mixture.route(logits, self.top, balance=self.balance)
        said = mixture.experts(y, ids, weights, self.w1.to(self.dtype), self.w2.to(self.dtype))
        return h + said.float(), ids

    def normals(self, features):
        return torch.nn.functional.normalize(features @ self.answer, dim=1)

    def class_losses(self, features, classes):
        """(n,) losses of the classes (n,) int32, the logits of all classes never kept."""
        return learning.cross_entropy(features.to(self.dtype), self.classes.to(self.dtype), classes)

    def forward(self, points):
        """(normals, ids): ids (n, top) are the experts that answered, best first."""
        features, ids = self.features(points)
        return self.normals(features), ids


def train(model, points, normals, steps: int, batch: int, rate=3e-3, balance_rate=3e-4, seed=2,
          classes=None, update="adam", orthogonal_rate=0.02):
    """Steps on random batches, the classes (n,) of the points with the normals if they are given;
    the balance moves after each.  update: "adam", or "orthogonal" for the matrices of the experts
    and of the classes."""
    matrices = [p for p in (model.w1, model.w2, model.classes)
                if update == "orthogonal" and p is not None]
    momenta = [torch.zeros_like(p) for p in matrices]
    opt = torch.optim.Adam([p for p in model.parameters()
                            if not any(p is m for m in matrices)], lr=rate)
    g = torch.Generator(device=points.device).manual_seed(seed)
    for _ in range(steps):
        at = torch.randint(points.shape[0], (batch,), generator=g, device=points.device)
        features, ids = model.features(points[at])
        loss = (model.normals(features) - normals[at]).square().sum(1).mean()
        if classes is not None:
            loss = loss + model.class_losses(features, classes[at]).mean()
        model.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        with torch.no_grad():
            for p, m in zip(matrices, momenta):
                if p.grad is not None:  # (the classes' is, where they are not learned)
                    learning.orthogonal_step(p, p.grad.contiguous(), m, orthogonal_rate, out=(p, m))
        counts = mixture.route_counts(ids, model.balance.numel())
        mixture.route_balance(counts, model.balance, balance_rate)


@torch.no_grad()
def mean_angle(model, points, normals) -> float:
    """Mean angle in degrees between the model's normals and the surface's."""
    cosine = (model(points)[0] * normals).sum(1).clamp(-1, 1)
    return torch.rad2deg(cosine.acos()).mean().item()


@torch.no_grad()
def right_classes(model, points, classes) -> dict:
    """Share of the points whose class has the largest logit: of the weights in 8 bits, and as they
    are."""
    features = model.features(points)[0].to(model.dtype)
    small = learning.linear_8bit(features, *learning.quantise(model.classes.detach()))
    full = features.float() @ model.classes.t()
    return {name: (logits.argmax(1) == classes).float().mean().item()
            for name, logits in (("right_in_8_bits", small), ("right", full))}


def run(units=64, dim=64, hidden=64, steps=300, batch=4096, n_points=20_000, seed=0,
        dtype=torch.bfloat16, classes=0, update="adam") -> dict:
    """Grows, trains and answers; returns what the command prints, and the model."""
    cloud = clouds.genus3_cloud(n_points, seed, jitter=0.0)
    points = torch.from_numpy(cloud).cuda()
    normals = torch.from_numpy(genus3_normals(cloud.astype(np.float64))).cuda()
    held = n_points // 5
    model = LocalExperts(grow_units(cloud, units), dim, hidden, dtype=dtype, seed=seed,
                         classes=classes)
    before = mean_angle(model, points[:held], normals[:held])
    nearest = nearest_units(grow_units(cloud, classes), points) if classes else None
    train(model, points[held:], normals[held:], steps, batch, update=update,
          classes=None if nearest is None else nearest[held:])
    after = mean_angle(model, points[:held], normals[:held])
    with torch.no_grad():
        ids = model(points[:held])[1]
        alone = [model(points[i:i + 1])[1][0].tolist() for i in range(4)]
    counts = mixture.route_counts(ids, units)
    got = {"experts": units, "angle_before": before, "angle_after": after,
           "pairs_most": int(counts.max()), "pairs_mean": ids.numel() / units,
           "experts_of_single_points": alone, "model": model}
    if classes:
        got.update(right_classes(model, points[:held], nearest[:held]))
    return got


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--units", type=int, default=64)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=64)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--classes", type=int, default=0)
    ap.add_argument("--update", choices=("adam", "orthogonal"), default="adam")
    got = run(**vars(ap.parse_args()))
    got.pop("model")
    print(json.dumps(got))


if __name__ == "__main__":
    main()
