"""The gradient of a row that is left out is zero, also where the weight is not
finite and the other rows' are NaN."""

import pytest
import torch

from tests.test_gpu_loss import LEFT_OUT, Case

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("x", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(5, 200), (40, 300), (64, 70), (70, 30), (400, 64), (70, 200), (300, 700)], ids=str)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_weight_that_is_not_finite(rows, classes, x, bad):
    c = Case([rows], 96, classes, x, x, F32, bias=True, weighted=True, seed=61)
    c.label[0][1] = LEFT_OUT
    c.label[0][2] = classes
    c.dloss[0][3] = 0.0
    c.w[0][classes // 2, 5] = bad
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert not c.dx[0][1:4].any()
    assert bool((c.loss[0][1:3] == 0).all())
    # (where bfloat16's infinity makes a logit of -infinity, the row has its other classes)
    others = c.x[0][:, 5] > 0
    others[1:4] = False
    assert bool(c.dx[0][others].isnan().all())
