"""The example that trains with layer norm, orthogonalised updates and the
elastic step together: its gradients against torch's own in binary64, and that
it learns."""

import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module")
def example():
    import orthogonal_elastic
    return orthogonal_elastic


def test_gradients_against_autograd(example):
    w = example.Workers(3, seed=4)
    for p in w.params:
        p.add_(torch.randn(p.shape, generator=w.gen, device=p.device) * 0.05)
    xs, ts = w.batches(130)
    w.gradients(xs, ts)
    for p, g, x, t in zip(w.params, w.grads, xs, ts):
        q = p.cpu().double().requires_grad_()
        w0, b0, A, w1, b1, B = example.views(q)
        norm = torch.nn.functional.layer_norm
        h = torch.relu(norm(x.cpu().double(), (example.WIDTH,), w0, b0) @ A)
        y = norm(h, (example.HIDDEN,), w1, b1) @ B
        ((y - t.cpu().double()) ** 2).mean().backward()
        # binary32 products and norms over at most 160 terms, twice: 1e-5 of
        # each tensor's gradient has a factor of ten to spare
        for got, want in zip(example.views(g.cpu().double()), example.views(q.grad)):
            assert float((got - want).norm()) <= 1e-5 * float(want.norm())


def test_it_learns(example):
    w = example.Workers(4, seed=1)
    losses = [float(w.step()) for _ in range(60)]
    assert all(l == l for l in losses)
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses
    spread = max(float((p - w.center).abs().max()) for p in w.params)
    assert spread < 1.0  # the workers stay around the center
