"""The cross entropy's gradients hold binary32 operands with 22 bits next to
their largest value, whatever the type of the result.

Where all logits of a row are equal and the classes a power of two, g is 1 / V,
and 1 / V - 1 for the label: values of 8 bits, which every form holds whole.  So

    dx = mean of the weight's rows - the label's row,   of values near one,

and dweight alike from the rows, is as good as its operand.  Bound: the computed
probabilities are off by the logits' logarithm and the exponential (4 + 2 |lse|
times 2^-22), and as much again where that is rounded away; operands by 2^-21;
sums of n terms in binary32 by n 2^-24, with 8 more for what is added to zeros;
the result is rounded once, half a step."""

import pytest
import torch

import paper_1801_03855_amd as tc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# rows and classes: few rows, few classes, and tiles
SIZES = [(3, 4), (40, 4), (2, 64), (64, 64), (70, 16), (3000, 32), (70, 128), (600, 1024),
         (4, 4), (8, 4), (128, 128), (256, 256), (512, 256)]  # (as many rows of each class: dweight is a difference too)


def near_one(*shape):
    return 1.0 + torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(41)) * 2.0 ** -11


def gradients(x, w, label, dw_type):
    rows = x.shape[0]
    loss, lse = [torch.empty(rows, device="cuda") for _ in range(2)]
    dx, dw = torch.empty_like(x), torch.empty(w.shape, dtype=dw_type, device="cuda")
    tc.cross_entropy([x], [w], None, [label], [loss], [lse])
    tc.cross_entropy_backward([x], [w], None, [label], [lse], None, [dx], [dw], None)
    torch.cuda.synchronize()
    g = torch.exp(-lse.double())[:, None].expand(rows, w.shape[0]).clone()
    dg = g * ((4 + 2 * lse.double().abs()) * 2.0 ** -22)[:, None]
    g[torch.arange(rows, device="cuda"), label] -= 1.0
    return dx.double(), dw.double(), g, 2 * dg


def check(got, want, size, d, terms, dtype, what):
    off = d + size * (2.0 ** -21 + (terms + 8) * 2.0 ** -24) + want.abs() * torch.finfo(dtype).eps / 2
    assert bool(((got - want).abs() <= off).all()), (what, float(((got - want).abs() / off).max()))


@pytest.mark.parametrize("rows,classes", SIZES, ids=str)
@pytest.mark.parametrize("cols", [64, 99])
@pytest.mark.parametrize("x_type", [BF16, F32], ids=["bf16", "f32"])
def test_the_weight_in_dx(rows, classes, cols, x_type):
    """Rows of zeros: their logits are zeros, whatever the weight."""
    w, label = near_one(classes, cols), torch.arange(rows, device="cuda") % classes
    dx, _, g, dg = gradients(torch.zeros(rows, cols, dtype=x_type, device="cuda"), w, label, F32)
    w = w.double()
    check(dx, g @ w, g.abs() @ w.abs(), dg @ w.abs(), classes, x_type, "dx")


@pytest.mark.parametrize("rows,classes", SIZES, ids=str)
@pytest.mark.parametrize("cols", [64, 99])
@pytest.mark.parametrize("dw_type", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("w_type", [BF16, F32], ids=["bf16", "f32"])
def test_the_rows_in_dweight(rows, classes, cols, w_type, dw_type):
    """A weight of zeros."""
    x, label = near_one(rows, cols), torch.arange(rows, device="cuda") % classes
    _, dw, g, dg = gradients(x, torch.zeros(classes, cols, dtype=w_type, device="cuda"), label, dw_type)
    x = x.double()
    check(dw, g.t() @ x, g.abs().t() @ x.abs(), dg.t() @ x.abs(), rows, dw_type, "dweight")
