"""The operators that a training step on this framework runs around the group's
average and elastic step, as cases that can be timed.

  norm       layer norm of K workers' rows, each worker with its own scale and
             shift: y, and the mean and 1 / deviation of every row
  norm_grad  its backward pass: the gradients of the rows, and of each worker's
             scale and shift (the sums over its rows)
  ortho      the momentum update of K workers' gradients of one tensor group,
             with every matrix of the group orthogonalised by five
             Newton-Schulz steps and every other tensor as it is

`own` false: the plain form, in elementary torch operations and 32 bits.
`own` true: the framework's calls.
"""

import functools
import math

import torch

own = False

EPS_NORM = 1e-5
EPS_ORTHO = 1e-7
MU = 0.95
STEPS = 5
A, B, C = 3.4445, -4.7750, 2.0315  # the quintic a x + b x^3 + c x^5 of each step

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    def norm(name, op, K, rows, cols, dtype, ragged=False, pad=0):
        return {"name": name, "op": op, "K": K, "rows": rows, "cols": cols, "dtype": dtype, "ragged": ragged, "pad": pad}

    def ortho(name, K, group, grad, out, momentum, layers=0, hidden=0, inner=0):
        return {"name": name, "op": "ortho", "K": K, "group": group, "grad": grad, "out": out, "momentum": momentum,
                "layers": layers, "hidden": hidden, "inner": inner}

    return [
        # One row a worker, as a model that answers takes them: latency.
        norm("norm_one_row", "norm", 2, 1, 512, "f32"),
        # A batch of odd width, views of wider rows, another number of rows for each worker.
        norm("norm_odd", "norm", 3, 3001, 1003, "f32", ragged=True, pad=5),
        # A large batch in bfloat16, eight workers: bandwidth.
        norm("norm_large", "norm", 8, 4096, 4096, "bf16"),
        # The backward pass of a handful of rows: latency.
        norm("norm_grad_few", "norm_grad", 2, 16, 512, "f32"),
        # Odd width, views, ragged: most of an ordinary batch's columns end inside a vector.
        norm("norm_grad_odd", "norm_grad", 4, 5003, 777, "f32", ragged=True, pad=3),
        # Few long rows.
        norm("norm_grad_wide", "norm_grad", 1, 2048, 16384, "bf16"),
        # The backward pass of the large batch.
        norm("norm_grad_large", "norm_grad", 8, 4096, 4096, "bf16"),
        # A toy model's group: three matrices of 10 to 32 rows.
        ortho("ortho_tiny", 2, "tiny", "f32", "f32", True),
        # The benchmark's group and workers, each worker with its momentum.
        ortho("ortho_resnet50", 8, "resnet50", "f32", "f32", True),
        # The averaged gradient of synchronous training: one copy, bfloat16 gradient and update.
        ortho("ortho_resnet50_mean", 1, "resnet50", "bf16", "bf16", True),
        # Square and 4:1 matrices of odd sizes, as a stack of equal layers has them, without momentum.
        ortho("ortho_layers", 2, "layers", "f32", "f32", False, 4, 1001, 4003),
        # The largest group: matrices of 4,096 rows, bfloat16.
        ortho("ortho_vgg16", 2, "vgg16", "bf16", "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "ortho"))
    if op != "ortho":
        K, cols = _log(rng, 1, 16), _log(rng, 64, 16384)
        rows = _log(rng, 1, min(32768, 1.3e8 / (K * cols)))
        cols = rng.choice((cols, (cols + 7) // 8 * 8, (cols + 63) // 64 * 64))
        return {"op": op, "K": K, "rows": rows + (rows == 3072), "cols": cols + (cols == 3072), "dtype": rng.choice(("f32", "bf16")),
                "ragged": rng.random() < 0.3 and rows > 8, "pad": rng.choice((0, 0, 0, 1, 8))}
    group = rng.choice(("tiny", "resnet50", "layers", "layers", "layers", "layers"))
    grad = rng.choice(("f32", "bf16"))
    case = {"op": op, "K": _log(rng, 1, 16 if group == "tiny" else 8), "group": group, "grad": grad,
            "out": rng.choice((grad, "f32")), "momentum": rng.random() < 0.7, "layers": 0, "hidden": 0, "inner": 0}
    if group == "layers":
        hidden = _log(rng, 16, 2048)
        hidden = rng.choice((hidden, (hidden + 15) // 16 * 16))
        inner = int(hidden * rng.choice((1.0, 2.0, 2.7, 4.0)))
        hidden, inner = hidden + (hidden == 3072), inner + (inner == 3072)
        # at most a third of the largest listed case's products
        most = 4e12 / (case["K"] * (4 * 20 * hidden ** 3 + 2 * (9 * inner * hidden ** 2 + 11 * hidden ** 3)))
        case |= {"layers": max(1, min(_log(rng, 1, 24), int(most))), "hidden": hidden, "inner": inner}
        if most < 1:
            case["K"] = 1
    return case


# ------------------------------------------------------------------- shapes

def _convolutions(rows):
    return [(o, i * k * k) for o, i, k in rows]


@functools.lru_cache(maxsize=8)
def _shapes_of(group, layers, hidden, inner):
    """The group's tensors in order: (rows, columns) of a matrix, (0, elements) of a vector."""
    if group == "tiny":
        return [(0, 64), (16, 144), (0, 16), (0, 16), (32, 144), (0, 32), (0, 32), (10, 32)]
    if group == "resnet50":
        out, cin = [(64, 147), (0, 64), (0, 64)], 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                for o, i in ((width, cin), (width, 9 * width), (4 * width, width)) + (((4 * width, cin),) if b == 0 else ()):
                    out += [(o, i), (0, o), (0, o)]
                cin = 4 * width
        return out + [(1000, 2048), (0, 1000)]
    if group == "vgg16":
        out, cin = [], 3
        for c in (64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512):
            out += [(c, 9 * cin), (0, c)]
            cin = c
        for i, o in ((25088, 4096), (4096, 4096), (4096, 1000)):
            out += [(o, i), (0, o)]
        return out
    layer = [(0, hidden), (0, hidden)] + [(hidden, hidden)] * 4 + [(0, hidden), (0, hidden), (inner, hidden), (hidden, inner)]
    return layer * layers


def _shapes(case):
    return _shapes_of(case["group"], case["layers"], case["hidden"], case["inner"])


def _numel(shape):
    return max(1, shape[0]) * shape[1]


@functools.lru_cache(maxsize=8)
def _places(group, layers, hidden, inner):
    """({(rows, columns): [first element of each matrix of that shape]}, [(first, elements) of each vector])."""
    at, matrices, vectors = 0, {}, []
    for shape in _shapes_of(group, layers, hidden, inner):
        if shape[0]:
            matrices.setdefault(shape, []).append(at)
        else:
            vectors.append((at, shape[1]))
        at += _numel(shape)
    return matrices, vectors


def _rows(case):
    K, rows = case["K"], case["rows"]
    return [max(1, rows * (k + 1) // K - k % 3) if case["ragged"] else rows for k in range(K)]


# ------------------------------------------------------------------- inputs

def _view(case, rows, gen, scale=1.0, shift=0.0):
    """[rows, cols] values in rows of cols + pad elements."""
    t = torch.randn(rows, case["cols"] + case["pad"], generator=gen, device="cuda").mul_(scale).add_(shift).to(_DT[case["dtype"]])
    return t[:, : case["cols"]]


def _empty(case, rows):
    return torch.empty(rows, case["cols"] + case["pad"], dtype=_DT[case["dtype"]], device="cuda")[:, : case["cols"]]


def _gradient(case, gen):
    """One worker's flat gradient: every matrix a product of few directions, as a batch leaves it, and noise."""
    parts = []
    for r, c in _shapes(case):
        g = torch.randn(max(1, r), c, generator=gen, device="cuda").mul_(0.004)
        if r:
            k = 1 + min(r, c) // 8
            g.addmm_(torch.randn(r, k, generator=gen, device="cuda"), torch.randn(k, c, generator=gen, device="cuda"),
                     alpha=0.01 / math.sqrt(k))
        parts.append(g.view(-1))
    return torch.cat(parts)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    K, s = case["K"], {"case": case}
    if case["op"] == "ortho":
        s["g"] = [_gradient(case, gen).to(_DT[case["grad"]]) for _ in range(K)]
        s["m"] = [_gradient(case, gen).mul_(4.0) for _ in range(K)] if case["momentum"] else None
        if own:
            import paper_1801_03855_amd as tc

            shapes = _shapes(case)
            s["group"] = tc.Group([_numel(h) for h in shapes])
            s["plan"] = tc.OrthoPlan(s["group"], K, [h if h[0] else None for h in shapes])
            s["out"] = [torch.empty(g.numel(), dtype=_DT[case["out"]], device="cuda") for g in s["g"]]
            s["workspace"] = torch.empty(tc.ortho_workspace(s["plan"]), dtype=torch.uint8, device="cuda")
        return s
    rows, cols = _rows(case), case["cols"]
    s["w"] = [torch.rand(cols, generator=gen, device="cuda").add_(0.5) for _ in range(K)]
    s["b"] = [torch.randn(cols, generator=gen, device="cuda").mul_(0.1) for _ in range(K)]
    s["x"] = [_view(case, r, gen, 1.5, 0.25) for r in rows]
    if case["op"] == "norm_grad":
        s["dy"] = [_view(case, r, gen, 0.01) for r in rows]
        s["mean"] = [x.float().mean(1) for x in s["x"]]
        s["rstd"] = [(x.float().var(1, unbiased=False) + EPS_NORM).rsqrt() for x in s["x"]]
    if own:
        import paper_1801_03855_amd as tc

        if case["op"] == "norm":
            s["y"] = [_empty(case, r) for r in rows]
            s["mean"] = [torch.empty(r, device="cuda") for r in rows]
            s["rstd"] = [torch.empty(r, device="cuda") for r in rows]
        else:
            s["dx"] = [_empty(case, r) for r in rows]
            s["dw"] = [torch.empty(cols, dtype=_DT[case["dtype"]], device="cuda") for _ in rows]
            s["db"] = [torch.empty(cols, dtype=_DT[case["dtype"]], device="cuda") for _ in rows]
            s["workspace"] = torch.empty(tc.layernorm_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------- plain forms

def _plain_norm(x, w, b):
    x = x.float()
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / x.shape[1] + EPS_NORM)
    return d * rstd[:, None] * w + b, mean, rstd


def _plain_norm_grad(dy, x, w, mean, rstd):
    dy, n = dy.float(), x.shape[1]
    xh = (x.float() - mean[:, None]) * rstd[:, None]
    h = dy * w
    dx = rstd[:, None] * (h - (h.sum(1) / n)[:, None] - xh * ((h * xh).sum(1) / n)[:, None])
    return dx, (dy * xh).sum(0), dy.sum(0)


def _newton_schulz(x):
    """[matrices, m, n], m <= n, each orthogonalised."""
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + EPS_ORTHO)
    for _ in range(STEPS):
        g = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.bmm(B * g + C * torch.bmm(g, g), x)
    return x


def _plain_ortho(gs, ms, places, dtype):
    gs = torch.stack(gs).float()
    if ms is not None:
        new = [m.mul_(MU).add_(g) for m, g in zip(ms, gs)]
        gs = gs + MU * torch.stack(new)
    out = gs.clone()  # what is no matrix stays as it is
    K = len(gs)
    for (r, c), at in places[0].items():
        x = torch.cat([gs[:, a : a + r * c] for a in at]).view(-1, r, c)
        x = _newton_schulz(x) if r <= c else _newton_schulz(x.transpose(1, 2).contiguous()).transpose(1, 2)
        for a, y in zip(at, x.reshape(len(at), K, r * c)):
            out[:, a : a + r * c] = y
    return list(out.to(dtype))


def run(s):
    case = s["case"]
    if case["op"] == "norm":
        if own:
            import paper_1801_03855_amd as tc

            tc.layernorm(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], EPS_NORM)
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        y, mean, rstd = zip(*[_plain_norm(x, w, b) for x, w, b in zip(s["x"], s["w"], s["b"])])
        return {"y": [v.to(_DT[case["dtype"]]) for v in y], "mean": mean, "rstd": rstd}
    if case["op"] == "norm_grad":
        if own:
            import paper_1801_03855_amd as tc

            tc.layernorm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["workspace"])
            return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
        got = [_plain_norm_grad(*v) for v in zip(s["dy"], s["x"], s["w"], s["mean"], s["rstd"])]
        return {k: [v[i].to(_DT[case["dtype"]]) for v in got] for i, k in enumerate(("dx", "dw", "db"))}
    if own:
        import paper_1801_03855_amd as tc

        tc.orthogonalize(s["plan"], s["g"], s["out"], s["m"], mu=MU, nesterov=True, steps=STEPS, coefficients=(A, B, C),
                         eps=EPS_ORTHO, workspace=s["workspace"])
        return {"out": s["out"], "m": s["m"]}
    places = _places(case["group"], case["layers"], case["hidden"], case["inner"])
    return {"out": _plain_ortho(s["g"], s["m"], places, _DT[case["out"]]), "m": s["m"]}


# ---------------------------------------------------------------- what it takes

def work(case):
    """Bytes: every input read once, every output written once.  Products:
    those of symmetric results count half, and two Newton-Schulz steps need one
    product of the matrix with itself (the polynomials in it commute), so that
    five steps of an m x n matrix, m <= n, need 9 m^2 n + 11 m^3 operations."""
    if case["op"] == "ortho":
        es = {"f32": 4, "bf16": 2}
        per = es[case["grad"]] + es[case["out"]] + (8 if case["momentum"] else 0)
        sides = [(min(h), max(h)) for h in _shapes(case) if h[0]]
        return {"bytes": case["K"] * per * sum(_numel(h) for h in _shapes(case)),
                "flops": case["K"] * sum(9 * m * m * n + 11 * m ** 3 for m, n in sides)}
    es, rows, cols, K = {"f32": 4, "bf16": 2}[case["dtype"]], sum(_rows(case)), case["cols"], case["K"]
    if case["op"] == "norm":
        return {"bytes": 2 * es * rows * cols + 8 * rows + 8 * K * cols, "flops": 8 * rows * cols}
    return {"bytes": 3 * es * rows * cols + 8 * rows + (4 + 2 * es) * K * cols, "flops": 14 * rows * cols}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        out = {"y": [], "mean": [], "rstd": []}
        for x, w, b in zip(s["x"], s["w"], s["b"]):
            x = x.double()
            mean, dev = x.mean(1), torch.sqrt(x.var(1, unbiased=False) + EPS_NORM)
            out["y"].append(torch.addcmul(b.double(), (x - mean[:, None]) / dev[:, None], w.double()))
            out["mean"].append(mean)
            out["rstd"].append(1 / dev)
        return out
    if case["op"] == "norm_grad":
        out = {"dx": [], "dw": [], "db": []}
        for dy, x, w, mean, rstd in zip(s["dy"], s["x"], s["w"], s["mean"], s["rstd"]):
            r = rstd.double()[:, None]
            xh, dy = x.double().sub_(mean.double()[:, None]).mul_(r), dy.double()
            out["dw"].append(torch.linalg.vecdot(dy, xh, dim=0))
            out["db"].append(dy.sum(0))
            h = dy.mul_(w.double())
            along = torch.linalg.vecdot(h, xh, dim=1)[:, None] / x.shape[1]
            out["dx"].append((h - h.mean(1, keepdim=True)).sub_(xh.mul_(along)).mul_(r))
        return out
    # X after t steps is p_t(X X^T) X with the product of the steps' polynomials, which commute
    out, momenta = [], [] if case["momentum"] else None
    matrices, _ = _places(case["group"], case["layers"], case["hidden"], case["inner"])
    for k in range(case["K"]):
        u = s["g"][k].double()
        if case["momentum"]:
            m = MU * s["m"][k].double() + u
            momenta.append(m)
            u = u + MU * m
        y = u.clone()
        for (r, c), places in matrices.items():
            for at in places:
                x = u[at : at + r * c].view(r, c)
                x = (x if r <= c else x.t()) / (torch.linalg.vector_norm(x) + EPS_ORTHO)
                gram = x @ x.t().contiguous()
                eye = torch.eye(len(gram), dtype=torch.float64, device="cuda")
                p, powers = eye, gram
                for _ in range(STEPS):
                    f = A * eye + powers @ (B * eye + C * powers)
                    p = f @ p
                    powers = f @ powers @ f
                x = p @ x
                y[at : at + r * c] = (x if r <= c else x.t()).reshape(-1)
        out.append(y)
    return {"out": out, "m": momenta}
