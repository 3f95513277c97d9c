"""The cross entropy's gradients of operands and factors of any size, each result
next to its own terms.  The bounds are those of tests/test_gpu_loss.py without
their absolute part, which hides results under 1e-30.  In its place stand steps of
binary32's smallest subnormal, which is what a sum under 2^-126 and each of its
terms are rounded to (of dweight f g, which the rows multiply), times what
multiplies the sum afterwards, and half a step of the result's own smallest."""

import pytest
import torch

from tests.test_gpu_loss import Case, eps, logits

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SMALLEST = {F32: 2.0 ** -150, BF16: 2.0 ** -134}  # half a step of the smallest subnormal


def gradients(c):
    """Of the only worker: ((name, result, formula, bound), ...)."""
    # (g of 11 bits, rounded to the nearest: half a step is 2^-11 of a value just over a power of two)
    n, bits = c.rows[0], lambda dtype: 2.0 ** -11 if dtype is BF16 else 2.0 ** -21
    x, w, lse = c.x[0].double(), c.w[0].double(), c.lse[0].double()[:, None]
    z, dz = logits(c, 0)
    f = c.dloss[0].double()[:, None] * c.scale
    p = torch.exp(z - lse)
    g = p.clone()
    g[torch.arange(n, device="cuda"), c.label[0]] -= 1.0
    dg = p * (2 * dz + ((z - lse).abs() + lse.abs() + 4) * 2.0 ** -22) + g.abs() * 2.0 ** -24 + 2.0 ** -38
    wide = lambda dtype: 0.0 if dtype is BF16 else 2.0 ** -21  # noqa: E731
    out = []
    fg, fdg = f * g, f.abs() * dg
    for name, got, want, size, d, operand, terms, rough in (
            ("dx", c.dx[0], f * (g @ w), f.abs() * (g.abs() @ w.abs()), f.abs() * (dg @ w.abs()), c.w[0].dtype, c.classes, f.abs()),
            ("dweight", c.dw[0], fg.t() @ x, fg.abs().t() @ x.abs(), fdg.t() @ x.abs(), c.x[0].dtype, n, c.scale * (1 + x.abs().amax(0))),
            ("dbias", c.db[0], fg.sum(0), fg.abs().sum(0), fdg.sum(0), BF16, n, c.scale)):
        off = d + size * (bits(got.dtype) + wide(operand) + (terms + 64) * 2.0 ** -24) + want.abs() * eps(got.dtype)
        out.append((name, got.double(), want, off + (terms + 16) * rough * 2.0 ** -149 + SMALLEST[got.dtype]))
    return out


SIZES = [(5, 200), (40, 300), (64, 70), (400, 30), (3000, 10), (70, 200), (300, 700)]


@pytest.mark.parametrize("rows,classes", SIZES, ids=str)
@pytest.mark.parametrize("small", [2.0 ** -120, 2.0 ** -112, 2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 112, 2.0 ** 120])
@pytest.mark.parametrize("x,dw", [(F32, F32), (BF16, F32), (F32, BF16)], ids=["f32", "bf16_rows", "bf16_dweight"])
def test_operands(rows, classes, small, x, dw):
    """A weight of values around `small`, and rows that make ordinary logits with it."""
    c = Case([rows], 80, classes, x, F32, dw, bias=True, weighted=True, seed=51)
    c.w[0].mul_(small)
    c.x[0].mul_(1.0 / small)
    run(c)


@pytest.mark.parametrize("rows,classes", SIZES, ids=str)
@pytest.mark.parametrize("small", [2.0 ** -118, 2.0 ** -90, 2.0 ** 90, 2.0 ** 118])
@pytest.mark.parametrize("x", [F32, BF16], ids=["f32", "bf16"])
def test_factors(rows, classes, small, x):
    """Every row's factor around `small`, and a scale that makes up for most of it."""
    c = Case([rows], 80, classes, x, x, F32, bias=True, weighted=True, seed=52, scale=0.25 * small ** -0.75)
    c.dloss[0].mul_(small)
    run(c)


def run(c):
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for name, got, want, off in gradients(c):
        assert float(want.abs().max()) > 100 * float(off.min()), name  # (or nothing would be compared)
        assert bool(((got - want).abs() <= off).all()), (name, float(((got - want).abs() / off).max()))


@pytest.mark.parametrize("rows,classes", SIZES, ids=str)
@pytest.mark.parametrize("order", ["first", "last", "in turn"])
@pytest.mark.parametrize("x", [F32, BF16], ids=["f32", "bf16"])
def test_small_next_to_large(rows, classes, order, x):
    """Rows and classes whose operands or factors are some 2^-95 or 2^-70 of the others', 32 at a time: nothing of them may
    count for more."""
    c = Case([rows], 80, classes, x, F32, F32, bias=True, weighted=True, seed=53)
    for t, by in ((c.x[0], 2.0 ** -95), (c.w[0], 2.0 ** -95), (c.dloss[0], 2.0 ** -70)):
        at = torch.arange(len(t), device="cuda")
        half = {"first": at < len(t) // 2, "last": at >= len(t) // 2, "in turn": at // 32 % 2 == 1}[order]
        t[half] *= by
    run(c)


def test_a_factor_of_zero_in_the_first_rows():
    c = Case([400], 80, 30, F32, F32, F32, bias=True, weighted=True, seed=54)
    c.dloss[0][:100] = 0.0
    c.dloss[0][100:164] *= 2.0 ** -80
    run(c)
