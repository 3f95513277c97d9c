"""The operators at the end of a training step's forward pass and the start of
its backward pass, as cases that can be timed.

  ce            softmax cross entropy of K workers' rows against each worker's
                own weight over the classes, without keeping the logits: every
                row's loss and log sum exp
  ce_grad       its backward pass: the gradients of the rows, and of each
                worker's weight and bias
  dropout       dropout of K workers' rows from a counter-based generator, and
                the residual added
  dropout_grad  its backward pass, the mask generated anew

`own` false: the plain form, in elementary torch operations and 32 bits.
`own` true: the framework's calls.
"""

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ES = {"f32": 4, "bf16": 2}
LEFT_OUT = -100  # the label of a row without one
SITE = 3


def listed():
    def ce(name, op, K, rows, cols, classes, x, w, dw="f32", bias=False, ragged=False, pad=0, weighted=False):
        return {"name": name, "op": op, "K": K, "rows": rows, "cols": cols, "classes": classes, "x": x, "w": w, "dw": dw,
                "bias": bias, "ragged": ragged, "pad": pad, "weighted": weighted}

    def drop(name, op, K, rows, cols, x, p, residual=False, ragged=False, pad=0):
        return {"name": name, "op": op, "K": K, "rows": rows, "cols": cols, "x": x, "p": p, "residual": residual,
                "ragged": ragged, "pad": pad}

    return [
        # One row a worker, 1,000 classes, as a single example is scored: latency.
        ce("ce_one_row", "ce", 2, 1, 512, 1000, "f32", "f32", bias=True),
        # The classifier of ResNet-50, 32 images a worker, eight workers.
        ce("ce_classes", "ce", 8, 32, 2048, 1000, "f32", "f32", bias=True),
        # A handful of rows over a large vocabulary: the weight's bandwidth.
        ce("ce_few_rows", "ce", 1, 8, 4096, 131072, "bf16", "bf16"),
        # Odd sizes, views of wider rows, rows left out, bfloat16 rows and binary32 parameters.
        ce("ce_odd", "ce", 3, 1501, 1003, 30011, "bf16", "f32", ragged=True, pad=5),
        # A large batch over a large vocabulary.
        ce("ce_large", "ce", 1, 8192, 4096, 131072, "bf16", "bf16"),
        # The backward pass of the last layer of VGG-16, 64 images a worker.
        ce("ce_grad_classes", "ce_grad", 4, 64, 4096, 1000, "f32", "f32", bias=True),
        # Odd sizes, bfloat16 rows, binary32 parameters and gradients, every row with its own factor.
        ce("ce_grad_odd", "ce_grad", 2, 901, 1003, 30011, "bf16", "f32", bias=True, ragged=True, pad=3, weighted=True),
        # The backward pass of the large batch, all in bfloat16.
        ce("ce_grad_large", "ce_grad", 1, 8192, 4096, 131072, "bf16", "bf16", "bf16"),
        # One row a worker of the width of VGG-16's fully connected layers: latency.
        drop("dropout_one_row", "dropout", 2, 1, 4096, "f32", 0.5),
        # A large batch with its residual, eight workers: bandwidth.
        drop("dropout_large", "dropout", 8, 4096, 4096, "bf16", 0.1, residual=True),
        # Rows of odd width, another number for each worker, views of wider rows.
        drop("dropout_grad_odd", "dropout_grad", 3, 3001, 1003, "f32", 0.2, ragged=True, pad=5),
        # The gradient of the large batch.
        drop("dropout_grad_large", "dropout_grad", 8, 4096, 4096, "bf16", 0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("ce", "ce_grad", "ce", "ce_grad", "dropout", "dropout_grad"))
    K = _log(rng, 1, 8)
    cols = _log(rng, 64, 8192 if op.startswith("ce") else 16384)
    cols = rng.choice((cols, (cols + 7) // 8 * 8, (cols + 63) // 64 * 64))
    case = {"op": op, "K": K, "cols": cols, "x": rng.choice(("f32", "bf16")), "pad": rng.choice((0, 0, 0, 1, 8))}
    if op.startswith("ce"):
        classes = _log(rng, 10, min(131072, 5e8 / (K * cols)))
        w = rng.choice((case["x"], "f32"))
        # at most the largest listed case's products, of which binary32 ones cost more
        most = (4e12 if case["x"] == w == "bf16" else 1e12) / (K * cols * classes)
        rows = _log(rng, 1, max(1, min(8192, most, 1e9 / (K * classes))))
        return case | {"rows": rows, "classes": classes, "w": w, "dw": rng.choice((w, "f32")), "bias": rng.random() < 0.4,
                       "ragged": rng.random() < 0.4 and rows > 8, "weighted": rng.random() < 0.5}
    rows = _log(rng, 1, min(32768, 1.3e8 / (K * cols)))
    return case | {"rows": rows, "p": rng.choice((0.1, 0.5, round(rng.uniform(0.01, 0.9), 3))),
                   "residual": op == "dropout" and rng.random() < 0.5, "ragged": rng.random() < 0.4 and rows > 8}


# ------------------------------------------------------------------- inputs

def _rows(case):
    K, rows = case["K"], case["rows"]
    return [max(1, rows * (k + 1) // K - k % 3) if case["ragged"] else rows for k in range(K)]


def _view(case, t):
    """The same values in rows of cols + pad elements, in the rows' type."""
    wide = torch.empty(t.shape[0], case["cols"] + case["pad"], dtype=_DT[case["x"]], device="cuda")
    wide[:, : case["cols"]] = t
    return wide[:, : case["cols"]]


def _empty(case, rows):
    return torch.empty(rows, case["cols"] + case["pad"], dtype=_DT[case["x"]], device="cuda")[:, : case["cols"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    rows, cols, s = _rows(case), case["cols"], {"case": case}
    if case["op"].startswith("dropout"):
        s["x"] = [_view(case, randn(r, cols)) for r in rows]
        s["residual"] = [_view(case, randn(r, cols) * 2.0) for r in rows] if case["residual"] else None
        s["random"] = torch.randint(0, 2 ** 62, (2,), generator=gen, device="cuda")  # the seed, and the step's number
        if own:
            s["y"] = [_empty(case, r) for r in rows]
        return s
    V, dt, wt = case["classes"], _DT[case["x"]], _DT[case["w"]]
    s["w"] = [(randn(V, cols) * cols ** -0.5).to(wt) for _ in rows]
    s["b"] = [(randn(V) * 0.1).to(wt) for _ in rows] if case["bias"] else None
    s["label"] = [torch.randint(0, V, (r,), generator=gen, device="cuda") for r in rows]
    s["x"] = []
    for w, label, r in zip(s["w"], s["label"], rows):
        # rows whose own class is a good guess, as training leaves them
        sure = torch.rand(r, 1, generator=gen, device="cuda") * 12.0
        s["x"].append(_view(case, randn(r, cols) * 1.5 + sure * w[label].float()))
        if case["ragged"]:
            label[torch.rand(r, generator=gen, device="cuda") < 0.1] = LEFT_OUT
    if case["op"] == "ce_grad":
        s["scale"] = 1.0 / max(rows)
        s["dloss"] = [torch.rand(r, generator=gen, device="cuda") + 0.5 for r in rows] if case["weighted"] else None
        s["lse"] = []
        for x, w, k in zip(s["x"], s["w"], range(case["K"])):
            z = x.float() @ w.float().t()
            s["lse"].append(torch.logsumexp(z if s["b"] is None else z.add_(s["b"][k].float()), 1))
            del z
    if own:
        import paper_1801_03855_amd as tc

        if case["op"] == "ce":
            s["loss"] = [torch.empty(r, device="cuda") for r in rows]
            s["lse"] = [torch.empty(r, device="cuda") for r in rows]
            need = tc.cross_entropy_workspace(rows, cols, V, dt, wt)
        else:
            dw = _DT[case["dw"]]
            s["dx"] = [_empty(case, r) for r in rows]
            s["dw"] = [torch.empty(V, cols, dtype=dw, device="cuda") for _ in rows]
            s["db"] = [torch.empty(V, dtype=dw, device="cuda") for _ in rows] if case["bias"] else None
            need = tc.cross_entropy_backward_workspace(rows, cols, V, dt, wt, dw)
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------- plain forms

def _logits(x, w, b):
    z = x.float() @ w.float().t()
    return z if b is None else z + b.float()


def _plain_ce(x, w, b, label):
    z = _logits(x, w, b)
    top = z.max(1).values
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    there = (label >= 0) & (label < w.shape[0])
    own_z = z[torch.arange(len(z), device=z.device), torch.where(there, label, 0)]
    return torch.where(there, lse - own_z, 0.0), lse


def _plain_ce_grad(x, w, b, label, lse, dloss, scale):
    G = torch.exp(_logits(x, w, b) - lse[:, None])
    there = (label >= 0) & (label < w.shape[0])
    at = torch.arange(len(G), device=G.device)
    G[at, torch.where(there, label, 0)] -= 1.0
    G *= torch.where(there, scale if dloss is None else scale * dloss, 0.0)[:, None]
    return G @ w.float(), G.t() @ x.float(), G.sum(0)


def _mul_hi_lo(a, m):
    """The halves of the 64-bit product of 32-bit words a (in 64-bit integers) and m."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    s = low + ((high & 0xFFFF) << 16)  # under 2^50
    return (high >> 16) + (s >> 32), s & 0xFFFFFFFF


def _philox(c, k0, k1):
    """Philox 4x32, 10 rounds (Salmon, Moraes, Dror and Shaw, 2011), of counters of four words."""
    for i in range(10):
        h0, l0 = _mul_hi_lo(c[0], 0xD2511F53)
        h1, l1 = _mul_hi_lo(c[2], 0xCD9E8D57)
        a, b = (k0 + i * 0x9E3779B9) & 0xFFFFFFFF, (k1 + i * 0xBB67AE85) & 0xFFFFFFFF
        c = (h1 ^ c[1] ^ a, l1, h0 ^ c[3] ^ b, l0)
    return c


def _keep(random, worker, rows, cols, p):
    """Where a worker's rows are kept: the words of one counter decide eight columns, 16 bits each."""
    seed, step, per = random[0], random[1], (cols + 7) // 8
    q = torch.arange(rows * per, device="cuda")
    c = (q & 0xFFFFFFFF, (q >> 32) | (worker << 16), (step & 0xFFFFFFFF).expand_as(q),
         (((step >> 32) & 0xFFFF) << 16 | SITE).expand_as(q))
    words = _philox(c, seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    u = torch.stack([h for v in words for h in (v & 0xFFFF, v >> 16)], 1).view(rows, per * 8)[:, :cols]
    return u >= _threshold(p)


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _plain_dropout(x, residual, keep, p):
    y = torch.where(keep, x.float() * (65536.0 / (65536 - _threshold(p))), 0.0)
    return y if residual is None else y + residual.float()


def run(s):
    case = s["case"]
    op, K, dt = case["op"], case["K"], _DT[case["x"]]
    if own:
        import paper_1801_03855_amd as tc

        if op == "ce":
            tc.cross_entropy(s["x"], s["w"], s["b"], s["label"], s["loss"], s["lse"], workspace=s["workspace"])
            return {"loss": s["loss"], "lse": s["lse"]}
        if op == "ce_grad":
            tc.cross_entropy_backward(s["x"], s["w"], s["b"], s["label"], s["lse"], s["dloss"], s["dx"], s["dw"], s["db"],
                                      scale=s["scale"], workspace=s["workspace"])
            return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
        if op == "dropout":
            tc.dropout(s["x"], s["residual"], s["y"], s["random"], site=SITE, p=case["p"])
        else:
            tc.dropout_backward(s["x"], s["y"], s["random"], site=SITE, p=case["p"])
        return {"y": s["y"]}
    bs = s["b"] if op.startswith("ce") and s["b"] is not None else [None] * K
    if op == "ce":
        got = [_plain_ce(*v) for v in zip(s["x"], s["w"], bs, s["label"])]
        return {"loss": [v[0] for v in got], "lse": [v[1] for v in got]}
    if op == "ce_grad":
        dl = s["dloss"] if s["dloss"] is not None else [None] * K
        out = {"dx": [], "dw": [], "db": [] if case["bias"] else None}
        for v in zip(s["x"], s["w"], bs, s["label"], s["lse"], dl):
            dx, dw, db = _plain_ce_grad(*v, s["scale"])
            out["dx"].append(dx.to(dt))
            out["dw"].append(dw.to(_DT[case["dw"]]))
            if case["bias"]:
                out["db"].append(db.to(_DT[case["dw"]]))
        return out
    res = s["residual"] or [None] * K
    return {"y": [_plain_dropout(x, r, _keep(s["random"], k, *x.shape, case["p"]), case["p"]).to(dt)
                  for k, (x, r) in enumerate(zip(s["x"], res))]}


# ---------------------------------------------------------------- what it takes

def work(case):
    """Bytes: every input read once, every output written once.  Products: the
    logits; backward the logits again, which are not kept, and the gradients of
    the rows and of the weight."""
    es, rows, cols, K = _ES[case["x"]], sum(_rows(case)), case["cols"], case["K"]
    if case["op"].startswith("dropout"):
        return {"bytes": (3 if case["residual"] else 2) * es * rows * cols + 16, "flops": 2 * rows * cols}
    V, ws = case["classes"], _ES[case["w"]]
    params = K * V * (cols + case["bias"])
    if case["op"] == "ce":
        return {"bytes": es * rows * cols + ws * params + 16 * rows, "flops": 2 * rows * cols * V}
    return {"bytes": 2 * es * rows * cols + (ws + _ES[case["dw"]]) * params + (12 + 4 * case["weighted"]) * rows,
            "flops": 6 * rows * cols * V}


def _exact_keep(random, worker, rows, cols, p):
    """The mask with 32-bit products taken in pieces of 16 bits, 10 rounds over an array of the four words."""
    seed, step = (int(v) for v in random)
    per = -(-cols // 8)
    n = rows * per
    w = torch.empty(4, n, dtype=torch.int64, device="cuda")
    w[0] = torch.arange(n, device="cuda") % 2 ** 32
    w[1] = torch.arange(n, device="cuda") // 2 ** 32 + worker * 2 ** 16
    w[2] = step % 2 ** 32
    w[3] = step // 2 ** 32 % 2 ** 16 * 2 ** 16 + SITE
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        parts = []
        for a, m in ((w[0], 0xD2511F53), (w[2], 0xCD9E8D57)):
            a0, a1, m0, m1 = a % 65536, a // 65536, m % 65536, m // 65536
            mid = a1 * m0 + a0 * m0 // 65536
            mid2 = a0 * m1 + mid % 65536
            parts += [a1 * m1 + mid // 65536 + mid2 // 65536, mid2 % 65536 * 65536 + a0 * m0 % 65536]
        w = torch.stack([parts[2] ^ w[1] ^ key[0], parts[3], parts[0] ^ w[3] ^ key[1], parts[1]])
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    u = torch.empty(n, 4, 2, dtype=torch.int64, device="cuda")
    u[:, :, 0], u[:, :, 1] = (w % 65536).t(), (w // 65536).t()
    return u.view(rows, per * 8)[:, :cols] >= round(p * 65536)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("dropout"):
        t, out = round(case["p"] * 65536), []
        for k, x in enumerate(s["x"]):
            y = _exact_keep(s["random"], k, *x.shape, case["p"]) * x.double() * 65536 / (65536 - t)
            out.append(y + s["residual"][k].double() if case["residual"] else y)
        return {"y": out}
    V, grad = case["classes"], case["op"] == "ce_grad"
    out = {"dx": [], "dw": [], "db": [] if case["bias"] else None} if grad else {"loss": [], "lse": []}
    for k in range(case["K"]):
        w = s["w"][k].double()
        b = s["b"][k].double() if case["bias"] else torch.zeros(V, dtype=torch.float64, device="cuda")
        parts = []
        dw, db = torch.zeros_like(w) if grad else None, torch.zeros_like(b)
        for at in range(0, _rows(case)[k], 1024):  # of rows
            x, label = s["x"][k][at : at + 1024].double(), s["label"][k][at : at + 1024]
            z = torch.addmm(b, x, w.t())
            hit = torch.nn.functional.one_hot(label.clamp(min=0), V).bool() & (label >= 0)[:, None]
            if not grad:
                lse = torch.logsumexp(z, 1)
                parts.append((((lse[:, None] - z) * hit).sum(1), lse))
                continue
            factor = s["scale"] * (label >= 0).double()
            if s["dloss"] is not None:
                factor = factor * s["dloss"][k][at : at + 1024].double()
            g = torch.exp(z.sub_(s["lse"][k][at : at + 1024].double()[:, None])).sub_(hit.double()).mul_(factor[:, None])
            parts.append((g @ w,))
            dw.addmm_(g.t(), x)
            db += g.sum(0)
        if grad:
            out["dx"].append(torch.cat([v[0] for v in parts]))
            out["dw"].append(dw)
            if case["bias"]:
                out["db"].append(db)
        else:
            out["loss"].append(torch.cat([v[0] for v in parts]))
            out["lse"].append(torch.cat([v[1] for v in parts]))
    return out
