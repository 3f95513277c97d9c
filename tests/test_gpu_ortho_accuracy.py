"""How far the orthogonalised update is from 64 bits, next to the same iteration
in binary32.

A binary32 iteration's error is what its products' sums and roundings leave,
carried through the steps that follow.  The kernels' products keep 22 bits of
their operands and sum in binary32, so their error is of the same kind: two
roundings of one thing, each an average over all elements and over three
matrices, which chance moves by less than a fifth.  A product that lost the
second half of an operand would be off by hundreds of times as much.
"""

import numpy as np
import pytest
import torch

from tests.test_gpu_ortho import CUBIC, check, flat, plan_for

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
QUINTIC = tuple(float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))
EPS = float(np.float32(1e-7))


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


def matrix(gen, shape, kind):
    """Few directions and noise, as a batch leaves a gradient, or noise alone."""
    r, c = shape
    g = torch.randn(r, c, generator=gen, device=DEV).mul_(0.004)
    if kind == "directions":
        k = 1 + min(r, c) // 8
        g.addmm_(torch.randn(r, k, generator=gen, device=DEV), torch.randn(k, c, generator=gen, device=DEV), alpha=0.01 / k ** 0.5)
    return g


def iterate(u, steps, dtype):
    """The formula in `dtype`, product by product."""
    x = u.to(dtype)
    x = x / (x.norm() + EPS)
    flip = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if flip else x
    a, b, c = QUINTIC
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if flip else x


def update(tc, us, dtype=torch.float32, steps=5):
    """One copy of a group of the matrices us."""
    plan = tc.OrthoPlan(tc.Group([u.numel() for u in us]), 1, [tuple(u.shape) for u in us])
    out = torch.empty(sum(u.numel() for u in us), dtype=dtype, device=DEV)
    tc.orthogonalize(plan, [torch.cat([u.reshape(-1) for u in us])], [out], steps=steps)
    return [p.view(u.shape) for p, u in zip(out.split([u.numel() for u in us]), us)]


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("steps", [1, 2, 5, 8])
@pytest.mark.parametrize("shapes", [[(65, 65)], [(100, 1000)], [(512, 512)], [(700, 1500), (130, 200), (40, 50)], [(256, 2304), (1000, 300)]])
def test_a_bfloat16_result_is_the_binary32_one_rounded(tc, shapes, steps):
    gen = generator(sum(map(sum, shapes)) + steps)
    for kind in ("directions", "gauss"):
        us = [matrix(gen, s, kind) for s in shapes]
        for wide, brief in zip(update(tc, us, steps=steps), update(tc, us, torch.bfloat16, steps)):
            assert torch.equal(wide.to(torch.bfloat16), brief)


@pytest.mark.parametrize("steps", [5, 8, 12, 24])
@pytest.mark.parametrize("shape", [(128, 512), (250, 400), (512, 512), (600, 1300)])
def test_a_bfloat16_result_after_many_steps(tc, shape, steps):
    """The rounding of the exact result, and twice a binary32 iteration's error
    (the steps do not contract: from 12 on the errors of both have grown a
    hundredfold, and chance with them)."""
    gen = generator(steps)
    for kind in ("directions", "gauss"):
        u = matrix(gen, shape, kind)
        want = iterate(u, steps, torch.float64)
        got = off(update(tc, [u], torch.bfloat16, steps)[0], want)
        assert got <= off(want.to(torch.bfloat16), want) + 2 * off(iterate(u, steps, torch.float32), want)


def no_further_than_binary32(tc, groups, seed, steps=5):
    """`groups` of matrices' shapes, whose update's error added up over three
    draws of each is at most a binary32 iteration's and a fifth, matrix by matrix."""
    gen = generator(seed)
    errs = [[0.0, 0.0] for _ in groups]
    for _ in range(3):
        us = [matrix(gen, s, "directions") for s in groups]
        for e, u, got in zip(errs, us, update(tc, us, steps=steps)):
            want = iterate(u, steps, torch.float64)
            e[0] += off(iterate(u, steps, torch.float32), want)
            e[1] += off(got, want)
    for s, (plain, ours) in zip(groups, errs):
        assert ours <= 1.2 * plain, f"{s}: {ours / 3:.2e} against {plain / 3:.2e}"


@pytest.mark.parametrize("shape", [(200, 20000), (128, 50000), (20000, 200), (255, 9000), (2000, 2100)])
def test_long_sums_of_one_step_at_a_time(tc, shape):
    no_further_than_binary32(tc, [shape], sum(shape))


@pytest.mark.parametrize("shape", [(200, 390), (255, 3000), (513, 600), (600, 1300), (1500, 700)])
def test_a_matrix_has_the_same_bits_whatever_its_neighbours(tc, shape):
    """Alone, next to matrices of another number of steps to a Gram matrix, and
    next to enough that tiles are larger and stages fewer."""
    gen = generator(sum(shape))
    u = matrix(gen, shape, "directions")
    alone, = update(tc, [u])
    for others in ([(600, 1300)], [(300, 310)], [(700, 1500), (1030, 1500)], [(512, 1152), (300, 300), (256, 2304)] * 12):
        for at in (0, len(others)):
            us = [matrix(gen, s, "gauss") for s in others]
            us.insert(at, u)
            assert torch.equal(update(tc, us)[at], alone), (others[:3], at)


@pytest.mark.parametrize("steps", [2, 5])
@pytest.mark.parametrize("shape", [(256, 512), (256, 2304), (600, 257), (300, 600), (300, 2000), (384, 768), (900, 448), (511, 1100),
                                   (512, 20000), (640, 30720), (768, 18432)])
def test_where_one_step_at_a_time_is_more_accurate(tc, shape, steps):
    no_further_than_binary32(tc, [shape], sum(shape) + steps, steps)


@pytest.mark.parametrize("steps", [2, 3, 5])
@pytest.mark.parametrize("shape", [(512, 1024), (512, 4608), (1030, 515), (768, 2304), (1024, 4096), (512, 8192),
                                   (1000, 8192), (1024, 65536), (1536, 20000)])
def test_matrices_that_take_two_steps_at_once(tc, shape, steps):
    no_further_than_binary32(tc, [shape], sum(shape) + steps, steps)


@pytest.mark.parametrize("triples", [[(0.0, 1.0, 0.0)], [(0.0, 1.5, -0.5), CUBIC], [(2.0, 0.0, -1.0), (0.0, 0.0, 1.0)],
                                     [CUBIC, (0.0, 1.0, 0.0), (0.0, 1.0, 0.0)], [QUINTIC] * 2, [QUINTIC] * 4])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_any_coefficients_of_two_steps_at_once(tc, triples, dtype):
    """Matrices of one and of two steps to a Gram matrix side by side, against
    the formula."""
    gen = torch.Generator().manual_seed(62)
    shapes = [(520, 1100), (511, 1023), 7, (30, 60), (1030, 513), (300, 200)]
    g = flat(gen, shapes, "one" if triples[0][0] != QUINTIC[0] else "directions", torch.float32)
    out = torch.empty_like(g, dtype=dtype)
    tc.orthogonalize(plan_for(tc, 1, shapes), [g], [out], steps=len(triples), coefficients=triples)
    check(out, g, shapes, triples)


@pytest.mark.parametrize("groups", [
    [(512, 1152), (300, 300), (256, 2304), (600, 1300)] * 12,   # 128 x 128 tiles, short sums: P X with one stage
    [(2000, 2100), (1500, 3100)],                                # 128 x 128 tiles, long sums: P X with two
    [(4096, 2000)], [(700, 5000), (1100, 600), (1001, 1003)], [(130, 512), (40, 50), (1024, 1024)],
])
def test_groups_that_take_every_kind_of_tile(tc, groups):
    """The formula's tests allow hundreds of roundings; these would show one
    operand without its second half."""
    no_further_than_binary32(tc, groups, 5 * len(groups))
