"""The operators around a layer's norms and a worker's gradients in one training loop: it runs, twice the same, and its gradients are
those of the same model in 64 bits.

Tolerance: the longest chains are sums over 1536 tokens and 192 entries in 32 bits through four matrices and two norms; each is within
its length times 2^-24 of the sum of magnitudes, together below 1e-4 of a tensor's norm where nothing cancels as a whole.
"""
import math
import os
import sys

import pytest
import torch

import paper_2302_07475_b200 as S  # noqa: F401

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_it_runs_and_repeats():
    import train_residual_classifier as example
    losses = example.train(steps=6, workers=5)
    assert all(math.isfinite(v) for v in losses)
    assert example.train(steps=3, workers=5) == losses[:3]


@pytest.mark.parametrize("max_norm", [1e9, 0.05])
def test_gradients_are_the_models(max_norm):
    import train_residual_classifier as example
    M, texts = 3, 64
    _, p = example.parameters(1, "cuda")
    p["table"].mul_(20)                                    # rows that the first norm's eps does not matter for
    for k in ("scale1", "shift1", "scale2", "shift2"):
        p[k].add_(torch.randn(p[k].shape, generator=torch.Generator("cuda").manual_seed(2), device="cuda") * 0.2)
    ids, labels = example.make_texts(M, texts, 5, "cuda")
    w = example.Workers(M, texts, "cuda")
    w.gradients(p, ids, labels, max_norm)
    first = w.grads.clone()
    w.gradients(p, ids, labels, max_norm)
    assert torch.equal(first, w.grads)

    def normed(t, scale, shift):
        c = t - t.mean(-1, keepdim=True)
        return c / torch.sqrt((c * c).mean(-1, keepdim=True) + example.EPS) * scale + shift

    for m in range(M):
        q = {k: v.detach().double().requires_grad_() for k, v in p.items()}
        there = (ids[m] >= 0).unsqueeze(-1)
        rows = torch.where(there, normed(q["table"][ids[m].clamp(min=0)], q["scale1"], q["shift1"]), 0.0)
        pooled = rows.sum(1) / there.sum(1)
        z = normed(pooled + torch.relu(pooled @ q["w1"].mT) @ q["w2"].mT, q["scale2"], q["shift2"])
        torch.nn.functional.cross_entropy(z @ q["w3"].mT, labels[m]).backward()
        norm = math.sqrt(sum(float(v.grad.square().sum()) for v in q.values()))
        assert abs(float(w.norm[m]) - norm) <= 1e-4 * norm
        c = min(1.0, max_norm / (norm + 1e-6))
        for k, v in q.items():
            have = w.parts[k][m].double()
            assert (have - c * v.grad.reshape(-1)).norm() <= 1e-4 * c * v.grad.norm(), k
