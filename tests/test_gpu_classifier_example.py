"""The example that trains with layer norm, dropout, cross entropy and the elastic
step together: its gradients against torch's own in binary64, and that it runs."""

import os
import sys

import pytest
import torch

from tests.philox import keep_mask

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module")
def example():
    import classifier_elastic
    return classifier_elastic


@pytest.mark.parametrize("rows", [40, 130])
def test_gradients_against_autograd(example, rows):
    w = example.Workers(3, seed=4)
    for p in w.params:
        p.add_(torch.randn(p.shape, generator=w.gen, device=p.device) * 0.05)
    w.random[1] = 2 ** 33 + 5
    xs, labels = w.batches(rows)
    loss = w.gradients(xs, labels)
    threshold, total = round(example.P * 65536), 0.0
    norm = torch.nn.functional.layer_norm
    for k, (p, g, x, t) in enumerate(zip(w.params, w.grads, xs, labels)):
        q, x = p.cpu().double().requires_grad_(), x.cpu().double()
        w0, b0, A, w1, b1, C, d = example.views(q)
        keep = torch.from_numpy(keep_mask(4, 2 ** 33 + 5, k, 0, rows, example.WIDTH, threshold))
        h = x + keep * (norm(x, (example.WIDTH,), w0, b0) @ A) * (65536 / (65536 - threshold))
        z = norm(h, (example.WIDTH,), w1, b1) @ C.t() + d
        own = torch.nn.functional.cross_entropy(z, t.cpu(), ignore_index=-1)
        own.backward()
        total += float(own.detach()) / 3
        # binary32 products and norms over at most 250 terms, three in a row: 1e-5 of
        # each tensor's gradient has a factor of ten to spare
        for got, want in zip(example.views(g.cpu().double()), example.views(q.grad)):
            assert float((got - want).norm()) <= 1e-5 * float(want.norm())
    assert abs(float(loss) - total) <= 1e-5 * total


def test_it_runs(example):
    w = example.Workers(4, seed=1)
    losses = [float(w.step()) for _ in range(10)]
    assert all(v == v and v < 100.0 for v in losses)
    assert all(bool(p.isfinite().all()) for p in w.params + [w.center])
    assert int(w.random[1]) == 10
