"""The cross entropy and its gradients against the formulas in 64 bits where the
tiled kernels have their large tiles, and classes in several pieces.  The bounds
are those of tests/test_gpu_loss.py; tests/test_loss_launches.py shows, without a
GPU, that these sizes take these kernels."""

import pytest
import torch

from tests.loss_tiles import TILES
from tests.test_gpu_loss import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("rows,cols,classes,x,w,dw,forward,backward", TILES, ids=str)
def test_tiles(rows, cols, classes, x, w, dw, forward, backward):
    """Ragged rows in wider ones, some left out, each with its own factor; labels on the first and last classes."""
    c = Case(rows, cols, classes, TYPES[x], TYPES[w], TYPES[dw], bias=True, weighted=True, out=0.1, pad=3, offset=1, seed=31)
    for label in c.label:
        label[:1] = classes - 1
        label[1:2] = 0
    c.forward()
    torch.cuda.synchronize()
    check_forward(c)
    if backward:
        c.backward()
        torch.cuda.synchronize()
        check_backward(c)
    first = [t.clone() for t in c.outputs()]
    for t in c.outputs() if backward else c.loss + c.lse:
        t.fill_(7.0)
    c.forward()
    if backward:
        c.backward()
    torch.cuda.synchronize()
    for a, b in zip(first, c.outputs()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,cols,classes,x", [((1 << 20) - 5, 67, 9001, "bf16"), (1 << 20, 64, 8200, "f32"), (131000, 4090, 50001, "bf16")], ids=str)
def test_pairs_joined_several_times(rows, cols, classes, x):
    """More rows and classes than the pairs have room for at a time.  Rows have nothing to do with each other, so 700 of them
    are compared, the first and last ones among them."""
    c = Case([rows], cols, classes, TYPES[x], TYPES[x], bias=True, out=0.1, seed=32)
    c.forward()
    torch.cuda.synchronize()
    some = torch.cat([torch.arange(64, device="cuda"), torch.randint(0, rows, (572,), device="cuda", generator=torch.Generator("cuda").manual_seed(1)),
                      torch.arange(rows - 64, rows, device="cuda")])
    c.rows = [len(some)]
    c.x, c.label, c.loss, c.lse = [[t[0][some]] for t in (c.x, c.label, c.loss, c.lse)]
    check_forward(c)
