"""K workers train a small layer-normed network by elastic averaging, with
orthogonalised momentum updates, on one GPU.

    python examples/orthogonal_elastic.py [--workers 4] [--steps 100]

Every worker holds the network's parameters as one flat buffer, its gradient as
another, and sees its own batches.  Per step and worker:

    a = norm(x; w0, b0);  h = relu(a A);  c = norm(h; w1, b1);  y = c B
    loss = mean (y - target)^2

  layernorm, layernorm_backward   both norms, on views of the flat buffers: the
                                  gradients of w and b land where the group
                                  expects them
  orthogonalize                   the momentum update; A and B (matrices of the
                                  group) are orthogonalised, w and b are not
  easgd_step                      every worker by its update, and the center
                                  toward the workers

The two matrix products of the network and their gradients are torch's.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1801_03855_amd as tc  # noqa: E402

WIDTH, HIDDEN, OUT = 96, 160, 24
# the network's tensors in the order of the flat buffers: w0, b0, A, w1, b1, B
SHAPES = [(WIDTH,), (WIDTH,), (WIDTH, HIDDEN), (HIDDEN,), (HIDDEN,), (HIDDEN, OUT)]


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
        # an orthogonalised update has singular values around 1 whatever the
        # gradient's size: scaled to elements of 0.2 or so on either side
        scales = [0.2 * max(s) ** 0.5 if len(s) == 2 else 1.0 for s in SHAPES]
        self.plan = tc.OrthoPlan(self.group, K, [s if len(s) == 2 else None for s in SHAPES], scales)
        n = self.group.numel
        start = torch.zeros(n, device=device)
        w0, b0, A, w1, b1, B = views(start)
        w0.fill_(1.0), w1.fill_(1.0)
        A.normal_(0.0, WIDTH ** -0.5, generator=gen), B.normal_(0.0, HIDDEN ** -0.5, generator=gen)
        self.params = [start.clone() for _ in range(K)]
        self.center = start.clone()
        self.grads, self.updates, self.momenta = [[torch.zeros(n, device=device) for _ in range(K)] for _ in range(3)]
        self.truth = torch.randn(WIDTH, OUT, generator=gen, device=device) * WIDTH ** -0.5

    def batches(self, rows):
        xs = [torch.randn(rows, WIDTH, generator=self.gen, device=self.device) * 2.0 + 0.5 for _ in range(self.K)]
        return xs, [torch.tanh(x @ self.truth) for x in xs]

    def norm(self, xs, w, b):
        """(y, mean, 1 / deviation) of every worker's rows."""
        ys = [torch.empty_like(x) for x in xs]
        means, rstds = [[torch.empty(x.shape[0], device=self.device) for x in xs] for _ in range(2)]
        tc.layernorm(xs, w, b, ys, means, rstds)
        return ys, means, rstds

    def gradients(self, xs, targets):
        """Every worker's gradient, into its flat buffer; the mean loss."""
        P = [views(p) for p in self.params]
        G = [views(g) for g in self.grads]
        w0, b0, A, w1, b1, B = zip(*P)
        gw0, gb0, gA, gw1, gb1, gB = zip(*G)
        a, mean0, rstd0 = self.norm(xs, w0, b0)
        z = [u @ m for u, m in zip(a, A)]
        h = [torch.relu(v) for v in z]
        c, mean1, rstd1 = self.norm(h, w1, b1)
        y = [u @ m for u, m in zip(c, B)]
        errors = [u - t for u, t in zip(y, targets)]
        dc = []
        for e, u, m, g in zip(errors, c, B, gB):
            dy = e * (2.0 / e.numel())
            torch.mm(u.t(), dy, out=g)
            dc.append(dy @ m.t())
        dh = [torch.empty_like(v) for v in h]
        tc.layernorm_backward(dc, h, w1, mean1, rstd1, dh, gw1, gb1)
        da = []
        for d, v, u, m, g in zip(dh, z, a, A, gA):
            dz = d * (v > 0)
            torch.mm(u.t(), dz, out=g)
            da.append(dz @ m.t())
        tc.layernorm_backward(da, xs, w0, mean0, rstd0, [torch.empty_like(x) for x in xs], gw0, gb0)
        return torch.stack([(e * e).mean() for e in errors]).mean()

    def step(self, rows=256, eta=0.02, rho=None):
        loss = self.gradients(*self.batches(rows))
        tc.orthogonalize(self.plan, self.grads, self.updates, self.momenta, mu=0.9)
        tc.easgd_step(self.group, self.params, self.updates, self.center, eta, 0.5 / (self.K * eta) if rho is None else rho)
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
