"""K workers train a small classifier by elastic averaging on one GPU: layer
norm, dropout with a residual, softmax cross entropy, and the elastic step.

    python examples/classifier_elastic.py [--workers 4] [--steps 100]

Every worker holds the network's parameters as one flat buffer, its gradient as
another, and sees its own batches.  Per step and worker:

    a = norm(x; w0, b0);  h = x + dropout(a A);  c = norm(h; w1, b1)
    loss = mean of cross_entropy(c C^T + d, label) over the rows with a label

  layernorm, layernorm_backward            both norms
  dropout, dropout_backward                the mask is made twice from the seed
                                           and the step, and never stored
  cross_entropy, cross_entropy_backward    the loss of every row, and the gradients
                                           of c, C and d; no logits
  easgd_step                               every worker by its gradient, and the
                                           center toward the workers

All work on views of the flat buffers, where the group expects the gradients.
The product with A and its gradients are torch's.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1801_03855_amd as tc  # noqa: E402

WIDTH, CLASSES, P = 96, 250, 0.2
# the network's tensors in the order of the flat buffers: w0, b0, A, w1, b1, C, d
SHAPES = [(WIDTH,), (WIDTH,), (WIDTH, WIDTH), (WIDTH,), (WIDTH,), (CLASSES, WIDTH), (CLASSES,)]


def views(flat):
    """The tensors of a flat buffer."""
    sizes = [torch.Size(s).numel() for s in SHAPES]
    return [v.view(s) for v, s in zip(flat.split(sizes), SHAPES)]


class Workers:
    def __init__(self, K, device="cuda", seed=0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.K, self.gen, self.device = K, gen, device
        self.group = tc.Group([torch.Size(s).numel() for s in SHAPES])
        n = self.group.numel
        start = torch.zeros(n, device=device)
        w0, b0, A, w1, b1, C, d = views(start)
        w0.fill_(1.0), w1.fill_(1.0)
        A.normal_(0.0, WIDTH ** -0.5, generator=gen), C.normal_(0.0, WIDTH ** -0.5, generator=gen)
        self.params = [start.clone() for _ in range(K)]
        self.center = start.clone()
        self.grads = [torch.zeros(n, device=device) for _ in range(K)]
        self.random = torch.tensor([seed, 0], dtype=torch.int64, device=device)  # the masks' seed and step
        self.means = torch.randn(CLASSES, WIDTH, generator=gen, device=device)

    def batches(self, rows):
        """Rows around their class's mean; one in eight has no label."""
        labels = [torch.randint(0, CLASSES, (rows,), generator=self.gen, device=self.device) for _ in range(self.K)]
        xs = [self.means[t] + torch.randn(rows, WIDTH, generator=self.gen, device=self.device) for t in labels]
        for t in labels:
            t[::8] = -1
        return xs, labels

    def norm(self, xs, w, b):
        """(y, mean, 1 / deviation) of every worker's rows."""
        ys = [torch.empty_like(x) for x in xs]
        means, rstds = [[torch.empty(x.shape[0], device=self.device) for x in xs] for _ in range(2)]
        tc.layernorm(xs, w, b, ys, means, rstds)
        return ys, means, rstds

    def gradients(self, xs, labels):
        """Every worker's gradient, into its flat buffer; the mean loss."""
        w0, b0, A, w1, b1, C, d = zip(*[views(p) for p in self.params])
        gw0, gb0, gA, gw1, gb1, gC, gd = zip(*[views(g) for g in self.grads])
        a, mean0, rstd0 = self.norm(xs, w0, b0)
        u = [v @ m for v, m in zip(a, A)]
        h = [torch.empty_like(x) for x in xs]
        tc.dropout(u, xs, h, self.random, p=P)
        c, mean1, rstd1 = self.norm(h, w1, b1)
        losses, lses = [[torch.empty(x.shape[0], device=self.device) for x in xs] for _ in range(2)]
        tc.cross_entropy(c, C, d, labels, losses, lses)
        # the mean over the rows with a label: their number stays on the GPU
        counts = [(t >= 0).sum() for t in labels]
        weights = [(1.0 / n).to(torch.float32).expand(len(t)).contiguous() for n, t in zip(counts, labels)]
        dc, dh, du, dx = [[torch.empty_like(x) for x in xs] for _ in range(4)]
        tc.cross_entropy_backward(c, C, d, labels, lses, weights, dc, gC, gd)
        tc.layernorm_backward(dc, h, w1, mean1, rstd1, dh, gw1, gb1)
        tc.dropout_backward(dh, du, self.random, p=P)
        da = []
        for g, v, m, out in zip(du, a, A, gA):
            torch.mm(v.t(), g, out=out)
            da.append(g @ m.t())
        tc.layernorm_backward(da, xs, w0, mean0, rstd0, dx, gw0, gb0)
        return torch.stack([t.sum() / n for t, n in zip(losses, counts)]).mean()

    def step(self, rows=200, eta=0.3, rho=None):
        self.random[1] += 1
        loss = self.gradients(*self.batches(rows))
        tc.easgd_step(self.group, self.params, self.grads, self.center, eta, 0.5 / (self.K * eta) if rho is None else rho)
        return loss


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    workers = Workers(a.workers)
    for i in range(a.steps):
        loss = workers.step()
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}: mean loss of {a.workers} workers {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
