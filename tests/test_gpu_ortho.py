"""The momentum update with orthogonalised matrices, against the formula in
binary64.

Tolerance.  A step's result X_j is off by a few roundings of its products:
operands of 22 bits or more, binary32 sums over n terms, so by
(32 + sqrt(n)) 2^-24 |X_j| in the Frobenius norm with room to spare, and by the
smallest step of a stored element, 2^-37 each at most.  What the remaining
steps make of a difference is at most its norm times the largest slope of their
composition over the singular values they can meet.  Adding that up over the
steps bounds the result; rounding it to bfloat16 adds 2^-8 of its norm.
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
QUINTIC = tuple(float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))
CUBIC = (1.5, -0.5, 0.0)
MU = float(np.float32(0.95))
EPS = float(np.float32(1e-7))


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


def formula(u, triples, eps=EPS):
    """(result, |X_0|, |X_1|, ...) of one matrix in binary64."""
    u = u.double()
    x = u / (u.norm() + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if flip else x
    norms = [float(x.norm())]
    for a, b, c in triples:
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
        norms.append(float(x.norm()))
    return (x.t() if flip else x), norms


def slopes(triples):
    """For every step, the largest slope of what follows it over the singular
    values it can meet (from [0, 1] at first)."""
    at = np.linspace(0, 1, 20001)
    after = []
    for i in range(len(triples) + 1):
        v, d = at.copy(), np.ones_like(at)
        for a, b, c in triples[i:]:
            d *= a + 3 * b * v ** 2 + 5 * c * v ** 4
            v = a * v + b * v ** 3 + c * v ** 5
        after.append(float(np.abs(d).max()))
        if i < len(triples):
            a, b, c = triples[i]
            top = float(np.abs(a * at + b * at ** 3 + c * at ** 5).max())
            at = np.linspace(0, top, 20001)
    return after


def tolerance(norms, triples, shape, dtype):
    m, n = sorted(shape)
    per = (32 + math.sqrt(n)) * U
    total = sum(s * (per * x + 2.0 ** -37 * math.sqrt(m * n)) for s, x in zip(slopes(triples), norms))
    return total + (2.0 ** -8 * norms[-1] if dtype == torch.bfloat16 else 0.0)


def check_matrix(got, u, triples, scale=1.0, what=""):
    want, norms = formula(u, triples)
    err = float((got.double() - scale * want).norm())
    tol = abs(scale) * tolerance(norms, triples, tuple(u.shape), got.dtype)
    assert math.isfinite(err) and err <= tol, f"{what}: off by {err:.3e}, at most {tol:.3e} allowed (norm {norms[-1]:.3e})"


def matrix(gen, shape, kind):
    r, c = shape
    g = torch.randn(r, c, generator=gen, dtype=torch.float64)
    if kind == "directions":
        k = 1 + min(r, c) // 8
        g = torch.randn(r, k, generator=gen, dtype=torch.float64) @ torch.randn(k, c, generator=gen, dtype=torch.float64) + 0.01 * g
    elif kind == "decay":
        s = torch.arange(1, min(r, c) + 1, dtype=torch.float64) ** -2.0
        a = torch.linalg.qr(torch.randn(r, min(r, c), generator=gen, dtype=torch.float64))[0]
        b = torch.linalg.qr(torch.randn(c, min(r, c), generator=gen, dtype=torch.float64))[0]
        g = (a * s) @ b.t()
    elif kind == "one":
        g = g[:, :1] * g[:1]
    elif kind == "orthogonal":
        q = torch.linalg.qr(torch.randn(max(r, c), min(r, c), generator=gen, dtype=torch.float64))[0]
        g = q if r >= c else q.t()
    return 0.01 * g


def size_of(shape):
    return shape if isinstance(shape, int) else shape[0] * shape[1]


def plan_for(tc, K, shapes, scales=None):
    group = tc.Group([size_of(s) for s in shapes])
    return tc.OrthoPlan(group, K, [None if isinstance(s, int) else s for s in shapes], scales)


def flat(gen, shapes, kind, dtype):
    parts = [matrix(gen, (1, s) if isinstance(s, int) else s, "gauss" if isinstance(s, int) else kind).reshape(-1) for s in shapes]
    return torch.cat(parts).to(dtype).to(DEV)


def pieces(buf, shapes):
    at = 0
    for s in shapes:
        n = size_of(s)
        yield s, buf[at:at + n] if isinstance(s, int) else buf[at:at + n].view(s)
        at += n


def check(out, u, shapes, triples, scales=None):
    """out against the update u (its exact values in any type)."""
    for i, ((s, got), (_, x)) in enumerate(zip(pieces(out.cpu(), shapes), pieces(u.cpu().double(), shapes))):
        f = 1.0 if scales is None else float(np.float32(scales[i]))
        if isinstance(s, int):
            bound = 4 * U * x.abs() + (2.0 ** -8 * x.abs() if out.dtype == torch.bfloat16 else 0.0)
            assert bool(((got.double() - f * x).abs() <= abs(f) * bound + 1e-38).all()), (i, s)
        elif size_of(s):
            check_matrix(got, x, triples, f, f"tensor {i} {s}")


ODD = [3, (1, 1), (1, 9), 1, (9, 1), (5, 3), (64, 147), 17, (33, 500), (0, 4), 0, (100, 63)]
MID = [(128, 128), 2, (129, 127), (257, 300), 5, (513, 64), (64, 576), (100, 1000)]


@pytest.mark.parametrize("g_dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                               (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("shapes", [ODD, MID])
@pytest.mark.parametrize("kind", ["gauss", "directions", "decay", "one", "orthogonal"])
def test_against_the_formula(tc, shapes, kind, g_dtype, out_dtype):
    gen = torch.Generator().manual_seed(len(shapes))
    shapes = [s for s in shapes if s != (0, 4)]
    gs = [flat(gen, shapes, kind, g_dtype) for _ in range(2)]
    outs = [torch.full_like(g, 7.0, dtype=out_dtype) for g in gs]
    tc.orthogonalize(plan_for(tc, 2, shapes), gs, outs)
    for g, o in zip(gs, outs):
        check(o, g, shapes, [QUINTIC] * 5)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("triple", [QUINTIC, CUBIC])
def test_every_number_of_steps(tc, steps, triple):
    gen = torch.Generator().manual_seed(steps)
    shapes = [(96, 200), 7, (140, 60), (20, 33)]
    g = flat(gen, shapes, "directions", torch.float32)
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=steps, coefficients=triple)
    check(out, g, shapes, [triple] * steps)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_and_square_matrices_together(tc, steps, dtype):
    """Matrices more than twice as long as wide take two steps to a product of
    the long side, square ones and narrow ones one: side by side, in both
    orientations and several copies, after every number of steps."""
    gen = torch.Generator().manual_seed(50 + steps)
    shapes = [(150, 310), 3, (145, 150), (420, 131), (40, 50), (100, 700), (257, 514)]
    gs = [flat(gen, shapes, kind, dtype) for kind in ("directions", "gauss", "decay")]
    outs = [torch.full_like(g, 7.0) for g in gs]
    tc.orthogonalize(plan_for(tc, 3, shapes), gs, outs, steps=steps)
    for g, o in zip(gs, outs):
        check(o, g, shapes, [QUINTIC] * steps)


@pytest.mark.parametrize("triples", [[(0.0, 1.0, 0.0)], [(0.0, 1.5, -0.5), CUBIC], [(2.0, 0.0, -1.0), (0.0, 0.0, 1.0), QUINTIC],
                                     [CUBIC, (0.0, 1.0, 0.0), (0.0, 1.0, 0.0)]])
def test_coefficients_that_are_zero(tc, triples):
    gen = torch.Generator().manual_seed(60)
    shapes = [(140, 300), (30, 60), (150, 160)]
    g = flat(gen, shapes, "one", torch.float32)
    out = torch.empty_like(g)
    if triples[0] == (2.0, 0.0, -1.0):
        # 2 x - x^5 reaches 1.27 on [0, 1], whose fifth power is 3.3, which the
        # quintic would make over 200
        with pytest.raises(tc.TCError):
            tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=len(triples), coefficients=triples)
        triples = triples[:2]
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=len(triples), coefficients=triples)
    check(out, g, shapes, triples)


@pytest.mark.parametrize("shape", [(64, 64), (64, 65), (63, 483), (64, 484), (64, 485), (64, 500), (65, 66), (1, 2500), (1, 2600),
                                   (16, 700), (17, 700), (2000, 16), (48, 180), (128, 128), (128, 129), (129, 258), (129, 257)])
def test_where_the_paths_meet(tc, shape):
    """Sizes around the limits of what a workgroup takes whole and of the tiles."""
    gen = torch.Generator().manual_seed(70)
    g = flat(gen, [2, shape, 1], "directions", torch.float32)
    for others in ([], [(200, 200)]):  # small matrices take another path next to large ones
        shapes = [2, shape, 1] + others
        u = torch.cat([g, flat(gen, others, "gauss", torch.float32)]) if others else g
        out = torch.empty_like(u)
        tc.orthogonalize(plan_for(tc, 1, shapes), [u], [out])
        check(out, u, shapes, [QUINTIC] * 5)


def test_coefficients_of_each_step(tc):
    gen = torch.Generator().manual_seed(77)
    shapes = [(150, 170), (40, 40)]
    triples = [QUINTIC, (2.0, -1.5, 0.5), CUBIC]
    g = flat(gen, shapes, "gauss", torch.float32)
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=3, coefficients=triples)
    check(out, g, shapes, triples)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
def test_momentum_and_scales(tc, nesterov, g_dtype):
    gen = torch.Generator().manual_seed(8)
    shapes = [5, (70, 90), 301, (131, 20), (10, 32)]
    scales = [1.0, 0.3, -2.0, 1.7, 0.0]
    gs = [flat(gen, shapes, "directions", g_dtype) for _ in range(3)]
    ms = [flat(gen, shapes, "gauss", torch.float32) for _ in range(3)]
    outs = [torch.empty_like(m) for m in ms]
    plan = plan_for(tc, 3, shapes, scales)
    for _ in range(2):
        before = [m.clone() for m in ms]
        tc.orthogonalize(plan, gs, outs, ms, mu=0.95, nesterov=nesterov)
        for g, m, old, o in zip(gs, ms, before, outs):
            want = MU * old.double() + g.double()
            assert bool(((m.double() - want).abs() <= 2 * U * (MU * old.double().abs() + g.double().abs())).all())
            check(o, g.double() + MU * m.double() if nesterov else m, shapes, [QUINTIC] * 5, scales)


def test_the_gradient_itself_as_the_place_of_the_update(tc):
    gen = torch.Generator().manual_seed(13)
    shapes = [9, (64, 200), (130, 130)]
    for dtype in (torch.float32, torch.bfloat16):
        g = flat(gen, shapes, "gauss", dtype)
        out = torch.empty_like(g)
        plan = plan_for(tc, 1, shapes)
        tc.orthogonalize(plan, [g], [out])
        tc.orthogonalize(plan, [g], [g])
        assert torch.equal(g, out)


@pytest.mark.parametrize("factor", [1e-3, 1e30, 1e36])
def test_the_gradient_s_scale_does_not_matter(tc, factor):
    gen = torch.Generator().manual_seed(14)
    shapes = [(60, 80), (200, 140)]
    g = flat(gen, shapes, "gauss", torch.float32) * factor
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out])
    check(out, g, shapes, [QUINTIC] * 5)


def test_zeros_and_values_that_are_not_finite_stay_in_their_matrix(tc):
    gen = torch.Generator().manual_seed(15)
    shapes = [(40, 50), (40, 50), (150, 160), (150, 160), (300, 20), 4]
    g = flat(gen, shapes, "gauss", torch.float32)
    parts = [p for _, p in pieces(g, shapes)]
    parts[0].zero_()
    parts[1][3, 4] = float("nan")
    parts[2][149, 0] = float("inf")
    parts[5][2] = float("-inf")
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out])
    got = [p for _, p in pieces(out, shapes)]
    assert float(got[0].abs().max()) == 0.0
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[2]).all())
    assert torch.equal(got[5], parts[5])
    for i in (3, 4):
        check_matrix(got[i].cpu(), parts[i].cpu(), [QUINTIC] * 5)


def test_a_large_matrix_of_each_orientation(tc):
    """Sums over 5,000 terms, tiles in both directions, and columns that end
    inside a tile."""
    gen = torch.Generator().manual_seed(16)
    shapes = [(700, 5000), (1100, 600), (1001, 1003)]
    g = flat(gen, shapes, "directions", torch.float32)
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out])
    check(out, g, shapes, [QUINTIC] * 5)


def test_many_copies_are_independent(tc):
    gen = torch.Generator().manual_seed(17)
    shapes = [(16, 144), 3, (130, 70)]
    K = 64
    gs = [flat(gen, shapes, "gauss", torch.bfloat16) for _ in range(K)]
    outs = [torch.empty_like(g, dtype=torch.float32) for g in gs]
    tc.orthogonalize(plan_for(tc, K, shapes), gs, outs)
    one = plan_for(tc, 1, shapes)
    alone = torch.empty_like(outs[0])
    for k in (0, 1, 31, 63):
        tc.orthogonalize(one, [gs[k]], [alone])
        assert torch.equal(alone, outs[k]), k


def test_a_group_without_matrices(tc):
    g = torch.randn(1000, device=DEV)
    out = torch.empty_like(g)
    plan = plan_for(tc, 1, [400, 0, 600], [2.0, 1.0, -1.0])
    tc.orthogonalize(plan, [g], [out])
    assert torch.equal(out, torch.cat([2 * g[:400], -g[400:]]))


def test_same_bits_again_on_another_stream_and_from_a_graph(tc):
    gen = torch.Generator().manual_seed(18)
    shapes = [(16, 144), 11, (200, 390), (64, 64), (500, 130)]
    gs = [flat(gen, shapes, "directions", torch.float32) for _ in range(2)]
    ms = [flat(gen, shapes, "gauss", torch.float32) for _ in range(2)]
    plan = plan_for(tc, 2, shapes)
    space = torch.empty(tc.ortho_workspace(plan), dtype=torch.uint8, device=DEV)
    first_m = [m.clone() for m in ms]
    first = [torch.empty_like(g) for g in gs]
    tc.orthogonalize(plan, gs, first, first_m)
    space.fill_(255)  # NaN in every format: nothing is read that was not written
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m2, out2 = [m.clone() for m in ms], [torch.empty_like(g) for g in gs]
    side.wait_stream(torch.cuda.current_stream())
    tc.orthogonalize(plan, gs, out2, m2, workspace=space, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(out2 + m2, first + first_m))
    out3 = [torch.empty_like(g) for g in gs]
    m3 = [m.clone() for m in ms]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tc.orthogonalize(plan, gs, out3, m3, workspace=space)
    for turn in range(3):
        for g in gs:
            g.mul_(1.25)
        want_m = [m.clone() for m in m3]
        want = [torch.empty_like(g) for g in gs]
        graph.replay()
        torch.cuda.synchronize()
        tc.orthogonalize(plan, gs, want, want_m)
        assert all(torch.equal(a, b) for a, b in zip(out3 + m3, want + want_m)), turn


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shapes,K", [([(512, 1152), (256, 2304), (512, 2048), (130, 512)] * 3, 8), ([(1030, 1500), (700, 2900)], 6),
                                      ([(2000, 2100)], 2), ([(300, 310)], 1)])
def test_same_bits_with_every_cu_at_work(tc, shapes, K, dtype):
    """Many tiles at once, again and again: a load into a buffer that another
    wave still reads would show as other bits now and then."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(90)
    n = sum(size_of(s) for s in shapes)
    gs = [torch.randn(n, generator=gen, device=DEV).to(dtype) for _ in range(K)]
    plan = plan_for(tc, K, shapes)
    first, again = [[torch.empty_like(g) for g in gs] for _ in range(2)]
    tc.orthogonalize(plan, gs, first)
    for _ in range(12):
        tc.orthogonalize(plan, gs, again)
        assert all(torch.equal(a, b) for a, b in zip(again, first))
    for s, got, u in ((s, a, b) for (s, a), (_, b) in zip(pieces(first[-1], shapes), pieces(gs[-1], shapes))):
        check_matrix(got.cpu(), u.cpu(), [QUINTIC] * 5)
        break


def test_flat_buffers_at_any_alignment(tc):
    gen = torch.Generator().manual_seed(19)
    shapes = [(64, 100), 3, (200, 141)]
    n = sum(size_of(s) for s in shapes)
    plan = plan_for(tc, 1, shapes)
    g = flat(gen, shapes, "gauss", torch.bfloat16)
    out = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    m = flat(gen, shapes, "gauss", torch.float32)
    m2 = m.clone()
    tc.orthogonalize(plan, [g], [out], [m])
    for shift in (1, 3):
        g2, o2, m3 = [torch.full((n + 8,), 7.0, dtype=t.dtype, device=DEV) for t in (g, out, m)]
        g2[shift:shift + n], m3[shift:shift + n] = g, m2
        tc.orthogonalize(plan, [g2[shift:shift + n]], [o2[shift:shift + n]], [m3[shift:shift + n]])
        assert torch.equal(o2[shift:shift + n], out) and torch.equal(m3[shift:shift + n], m)
        for t in (o2, m3):
            assert float(t[:shift].float().min()) == 7.0 and float(t[shift + n:].float().min()) == 7.0


@pytest.mark.parametrize("steps", [2, 4, 5])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_around_the_sizes_that_take_two_steps_at_once(tc, steps, dtype):
    gen = torch.Generator().manual_seed(19)
    shapes = [(255, 600), (256, 512), (511, 256), (257, 514), (600, 257), (300, 599), (1300, 300)]
    triples = [QUINTIC] * steps
    us = [flat(gen, shapes, "directions", torch.float32)]
    outs = [torch.full((us[0].numel(),), 7.0, dtype=dtype, device=DEV)]
    tc.orthogonalize(plan_for(tc, 1, shapes), us, outs, steps=steps, coefficients=triples)
    check(outs[0], us[0], shapes, triples)


@pytest.mark.parametrize("triples", [[(0.0, 1.0, 0.0)], [(0.0, 1.5, -0.5), CUBIC], [(2.0, 0.0, -1.0), (0.0, 0.0, 1.0)],
                                     [CUBIC, (0.0, 1.0, 0.0), (0.0, 1.0, 0.0)]])
def test_zero_coefficients_of_two_steps_at_once(tc, triples):
    gen = torch.Generator().manual_seed(61)
    shapes = [(260, 600), (30, 60), (520, 256)]
    g = flat(gen, shapes, "one", torch.float32)
    out = torch.empty_like(g)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=len(triples), coefficients=triples)
    check(out, g, shapes, triples)


@pytest.mark.parametrize("shape", [(64, 200), (128, 512), (129, 258), (516, 129), (160, 640), (200, 1000), (255, 600), (300, 400)])
def test_as_accurate_as_a_binary32_iteration(tc, shape):
    """No further from 64 bits than the same steps in binary32, and a fifth of
    that for what is chance (the errors of two roundings of one thing, each an
    average over all elements)."""
    gen = torch.Generator().manual_seed(sum(shape))
    errs = [0.0, 0.0]
    for _ in range(3):
        u = matrix(gen, shape, "directions").to(torch.float32)
        want, norms = formula(u, [QUINTIC] * 5)
        x = u / (u.norm() + EPS)
        x = x.t().contiguous() if shape[0] > shape[1] else x
        for a, b, c in [QUINTIC] * 5:
            g = x @ x.t().contiguous()
            x = a * x + (b * g + c * (g @ g)) @ x
        x = x.t() if shape[0] > shape[1] else x
        out = torch.empty(u.numel(), device=DEV)
        tc.orthogonalize(plan_for(tc, 1, [shape]), [u.reshape(-1).to(DEV)], [out])
        for i, got in enumerate((x, out.view(shape).cpu())):
            errs[i] += float((got.double() - want).norm()) / norms[-1]
    assert errs[1] <= 1.2 * errs[0], f"{errs[1] / 3:.2e} against {errs[0] / 3:.2e}"


def test_refusals(tc):
    group = tc.Group([6, 20])

    def refused(kind, fn, *a, **kw):
        with pytest.raises(kind):
            fn(*a, **kw)

    refused(tc.TCError, tc.OrthoPlan, group, 1, [(2, 4), None])
    refused(tc.TCError, tc.OrthoPlan, group, 1, [(-2, -3), None])
    refused(tc.TCError, tc.OrthoPlan, group, 1, [(0, 6), None])
    refused(tc.TCError, tc.OrthoPlan, group, 0, [None, None])
    refused(tc.TCError, tc.OrthoPlan, group, 65, [None, None])
    refused(tc.TCError, tc.OrthoPlan, group, 1, [None, None], [1.0, float("inf")])
    refused(tc.TCError, tc.OrthoPlan, tc.Group([(1 << 22) + 1]), 1, [(1, (1 << 22) + 1)])
    refused(ValueError, tc.OrthoPlan, group, 1, [None])
    refused(ValueError, tc.OrthoPlan, group, 1, [None, None], [1.0])
    plan = tc.OrthoPlan(group, 2, [(2, 3), (4, 5)])
    gs = [torch.ones(26, device=DEV) for _ in range(2)]
    outs = [torch.zeros(26, device=DEV) for _ in range(2)]
    ms = [torch.ones(26, device=DEV) for _ in range(2)]
    call = tc.orthogonalize
    refused(ValueError, call, plan, gs[:1], outs)
    refused(ValueError, call, plan, gs, outs, ms[:1])
    refused(TypeError, call, plan, [g.half() for g in gs], outs)
    refused(TypeError, call, plan, gs, outs, [m.bfloat16() for m in ms])
    refused(ValueError, call, plan, [g[:25] for g in gs], outs)
    refused(ValueError, call, plan, gs, outs, coefficients=[(1.0, 0.0, 0.0)] * 4)
    refused(tc.TCError, call, plan, gs, outs, steps=0, coefficients=[QUINTIC][:0] or QUINTIC)
    refused(tc.TCError, call, plan, gs, outs, steps=65)
    refused(tc.TCError, call, plan, gs, outs, eps=0.0)
    refused(tc.TCError, call, plan, gs, outs, mu=float("nan"))
    refused(tc.TCError, call, plan, gs, outs, coefficients=(float("inf"), 0.0, 0.0))
    refused(tc.TCError, call, plan, gs, outs, coefficients=(5.0, 0.0, 0.0))
    refused(tc.TCError, call, plan, gs, outs, coefficients=(20.0, -19.5, 0.0), steps=1)
    refused(tc.TCError, call, plan, gs, [outs[0], outs[0]])
    refused(tc.TCError, call, plan, gs, [gs[1], outs[1]])
    refused(tc.TCError, call, plan, gs, outs, [ms[0], gs[0]])
    # a matrix of 100 rows needs a workspace (those of the first plan fit a workgroup's own memory)
    assert tc.ortho_workspace(plan) == 0
    large = tc.OrthoPlan(tc.Group([100 * 120]), 1, [(100, 120)])
    g1, o1 = torch.ones(12000, device=DEV), torch.zeros(12000, device=DEV)
    refused(tc.TCError, call, large, [g1], [o1], workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
    big = torch.zeros(tc.ortho_workspace(large) + 512, dtype=torch.uint8, device=DEV)
    refused(tc.TCError, call, large, [g1], [o1], workspace=big[8:])
    refused(tc.TCError, call, large, [g1], [big[:48000].view(torch.float32)], workspace=big)
    refused(ValueError, call, large, [g1], [o1], workspace=big.cpu())
    assert float(o1.abs().max()) == 0.0
    assert all(float(o.abs().max()) == 0.0 for o in outs)
    assert tc.lib().tc_orthogonalize(None, None, 0, None, 0.9, 0, None, 0, 1, None, 1e-7, None, 0, None) == tc.TC_EINVAL
    assert not tc.lib().tc_ortho_create(None, 1, None, None, None)
    assert tc.lib().tc_ortho_workspace(None) == -1
    tc.lib().tc_ortho_destroy(None)
    call(plan, gs, outs, ms)
    call(large, [g1], [o1], workspace=big)
