"""Dropout of K workers' rows: the mask bit for bit against Philox in numpy, the
values against the formula in 64 bits."""

import numpy as np
import pytest
import torch

import paper_1801_03855_amd as tc
from tests.philox import keep_mask

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def view(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def random(seed=1234567890123456789, step=98765432101234):
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def want(x, residual, worker, site, p, seed=1234567890123456789, step=98765432101234):
    """(values in 64 bits, how far a binary32 product and sum, rounded once to the type, may be)."""
    t = threshold(p)
    keep = torch.from_numpy(keep_mask(seed, step, worker, site, x.shape[0], x.shape[1], t))
    scaled = torch.where(keep, x.double().cpu() * (65536 / (65536 - t) if t < 65536 else 0.0), 0.0)
    y = scaled + (0.0 if residual is None else residual.double().cpu())
    half = torch.finfo(x.dtype).eps / 2
    return keep, y, y.abs() * (half + 2.0 ** -24) + scaled.abs() * 2.0 ** -22


def check(rows, cols, dtype, p=0.3, residual=False, pad=0, in_place=None, site=5):
    gen = torch.Generator(device="cuda").manual_seed(0)
    xs = [view(torch.randn(r, cols, generator=gen, device="cuda").to(dtype), pad) for r in rows]
    rs = [view(torch.randn(r, cols, generator=gen, device="cuda").to(dtype), pad) for r in rows] if residual else None
    expected = [want(x, None if rs is None else rs[k], k, site, p) for k, x in enumerate(xs)]
    ys = xs if in_place == "x" else rs if in_place == "residual" else [view(torch.zeros_like(x), pad) for x in xs]
    tc.dropout(xs, rs, ys, random(), site=site, p=p)
    torch.cuda.synchronize()
    for y, (keep, ref, off) in zip(ys, expected):
        assert bool(((y.double().cpu() - ref).abs() <= off).all())
        if rs is None:
            assert not y.cpu()[~keep].any()
    return expected


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [([1], 1), ([1, 1], 8), ([2, 0, 3], 7), ([5], 12), ([33, 1], 1003), ([4, 9], 4096), ([300], 72),
                                       ([1], 16385), ([700, 650], 260)], ids=str)
@pytest.mark.parametrize("residual,pad", [(False, 0), (True, 5)])
def test_sizes(rows, cols, dtype, residual, pad):
    check(rows, cols, dtype, residual=residual, pad=pad)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 0.1, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_probabilities(p, dtype):
    for keep, _, _ in check([64], 1000, dtype, p=p):
        n, q = keep.numel(), 1 - threshold(p) / 65536
        # five deviations of a binomial count
        assert abs(int(keep.sum()) - n * q) <= 5 * (n * q * (1 - q)) ** 0.5


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cols", [96, 101, 3])
@pytest.mark.parametrize("place", ["x", "residual"])
def test_in_place(dtype, cols, place):
    check([50, 7], cols, dtype, residual=place == "residual", pad=3, in_place=place)


def test_all_workers():
    check([3] * 64, 24, F32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cols", [96, 101])
def test_gradient_has_the_same_mask(dtype, cols):
    """dx = the factor of y = drop(x) times dy; of ones, so that y is the factor itself."""
    rows, p = [70, 9], 0.4
    ones = [torch.ones(r, cols, dtype=dtype, device="cuda") for r in rows]
    dys = [torch.randn(r, cols, device="cuda").to(dtype) for r in rows]
    ys, dxs = [[torch.empty_like(t) for t in ones] for _ in range(2)]
    tc.dropout(ones, None, ys, random(), site=9, p=p)
    tc.dropout_backward(dys, dxs, random(), site=9, p=p)
    torch.cuda.synchronize()
    factor = 65536 / (65536 - threshold(p))
    for y, dy, dx in zip(ys, dys, dxs):
        ref = torch.where(y != 0, dy.double() * factor, 0.0)
        assert bool(((dx.double() - ref).abs() <= ref.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -22)).all())


@pytest.mark.parametrize("cols", [64, 61])
def test_what_is_dropped_may_hold_anything(cols):
    for bad in (float("nan"), float("inf")):
        x = torch.randn(40, cols, device="cuda")
        keep, ref, off = want(x, None, 0, 0, 0.5)
        x[~keep.cuda()] = bad
        y = torch.empty_like(x)
        tc.dropout([x], None, [y], random(), p=0.5)
        torch.cuda.synchronize()
        assert bool(((y.double().cpu() - ref).abs() <= off).all())


def test_seed_step_and_site_each_change_the_mask():
    x, masks = torch.ones(64, 64, device="cuda"), []
    for seed, step, site in ((1, 1, 0), (2, 1, 0), (1 + 2 ** 40, 1, 0), (1, 2, 0), (1, 1 + 2 ** 33, 0), (1, 1, 1), (-1, 1, 0), (1, 1, 65535)):
        y = torch.empty_like(x)
        tc.dropout([x], None, [y], random(seed, step), site=site, p=0.5)
        torch.cuda.synchronize()
        assert np.array_equal((y != 0).cpu().numpy(), keep_mask(seed, step, 0, site, 64, 64, 32768))
        masks.append(y != 0)
    for i in range(len(masks)):
        for j in range(i):
            # two masks of 4,096 fair places agree in half of them, within five deviations
            assert abs(int((masks[i] == masks[j]).sum()) - 2048) <= 5 * 32


def test_a_replayed_graph_reads_the_step_anew():
    x, y = torch.ones(32, 40, device="cuda"), torch.empty(32, 40, device="cuda")
    state = random(7, 0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tc.dropout([x], None, [y], state, p=0.5)
    for step in range(3):
        state[1] = step
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal((y != 0).cpu().numpy(), keep_mask(7, step, 0, 0, 32, 40, 32768))


def test_another_stream():
    x = torch.randn(300, 1000, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    state = random()
    tc.dropout([x], None, [a], state)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    tc.dropout([x], None, [b], state, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_more_than_32_bits_of_bytes():
    """A row stride that puts the last row past 4 GiB."""
    rows, cols, ld = 70000, 16, 40000
    buf = torch.empty(rows * ld, dtype=BF16, device="cuda")
    x = buf.view(rows, ld)[:, :cols]
    x.copy_(torch.randn(rows, cols, device="cuda"))
    y = torch.empty(rows, cols, dtype=BF16, device="cuda")
    tc.dropout([x], None, [y], random(), p=0.25)
    torch.cuda.synchronize()
    keep, ref, off = want(x, None, 0, 0, 0.25)
    assert bool(((y.double().cpu() - ref).abs() <= off).all())
