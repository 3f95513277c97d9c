"""The layer norm's buffers in places next to each other and in each other."""

import pytest
import torch

from tests.test_gpu_norm import DEV, check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


def test_all_in_the_rows_of_one_buffer(tc):
    """x, y, dy and dx next to each other in the rows of one buffer, and the
    scale, shift, statistics, their gradients and the workspace between them."""
    rows, cols = 6, 40
    need = tc.layernorm_workspace([rows], cols)
    wide = 8 * cols + max(need // 4 + 64, 512)
    buf = torch.full((rows, wide), float("nan"), device=DEV)
    (x0,), (dy0,), (w0,), (b0,) = make(torch.Generator().manual_seed(1), [rows], cols, torch.float32)
    x, y, dy, dx = [buf[:, i * cols:(i + 1) * cols] for i in range(4)]
    w, b, dw, db = [buf[i, 4 * cols:5 * cols] for i in range(4)]
    mean, rstd = buf[4, 4 * cols:4 * cols + rows], buf[5, 4 * cols:4 * cols + rows]
    space = buf[2, 8 * cols:8 * cols + need // 4 + 4]
    skip = -space.data_ptr() % 16 // 4
    space = space[skip:skip + need // 4]
    x.copy_(x0), dy.copy_(dy0), w.copy_(w0), b.copy_(b0)
    tc.layernorm([x], [w], [b], [y], [mean], [rstd])
    check_forward(x0, w0, b0, y, mean, rstd, 1e-5)
    tc.layernorm_backward([dy], [x], [w], [mean], [rstd], [dx], [dw], [db], space)
    check_backward(dy0, x0, w0, mean, rstd, dx, dw, db)
    assert torch.equal(x, x0) and torch.equal(dy, dy0) and torch.equal(w, w0)


def test_refusals(tc):
    (x,), (dy,), (w,), (b,) = make(torch.Generator().manual_seed(2), [6], 40, torch.float32)
    y, dx, dw, db = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)
    mean, rstd = torch.zeros(6, device=DEV), torch.ones(6, device=DEV)
    for args in ([[x], [w], [b], [y], [y[1, :6]], [rstd]], [[x], [w], [b], [y], [mean], [mean]], [[x], [y[0]], [b], [y], [mean], [rstd]],
                 [[x], [w], [b], [y], [w[:6]], [rstd]], [[x], [w], [y[5]], [y], [mean], [rstd]]):
        with pytest.raises(tc.TCError):
            tc.layernorm(*args)
    space = torch.empty(tc.layernorm_workspace([6], 40), dtype=torch.uint8, device=DEV)
    inside = torch.zeros(space.numel() + 6 * 40 * 4, dtype=torch.uint8, device=DEV)
    last = inside[-6 * 40 * 4 - 16:-16].view(torch.float32).view(6, 40)
    tail = torch.zeros(40, device=DEV)
    for args in ([[dy], [x], [w], [tail[:6]], [rstd], [dx], [tail], [db], space], [[dy], [x], [w], [mean], [tail[-6:]], [dx], [dw], [tail], space],
                 [[dy], [last], [w], [mean], [rstd], [dx], [dw], [db], inside], [[dy], [x], [w], [mean], [rstd], [last], [dw], [db], inside],
                 [[dy], [x], [dx[2]], [mean], [rstd], [dx], [dw], [db], space], [[dy], [x], [w], [dx[0, :6]], [rstd], [dx], [dw], [db], space]):
        with pytest.raises(tc.TCError):
            tc.layernorm_backward(*args)
    for t in (y, dx, dw, db, mean, tail):
        assert float(t.abs().max()) == 0.0
