"""Layer norm of K workers' rows and its backward pass, against the formulas in
binary64.

Tolerances follow from the arithmetic.  With u = 2^-24, a row's sums are chains
of at most c = 64 + cols / 128 binary32 additions (up to 32 elements a lane, or
cols / 1,024 vectors of 8 of them on long rows, then trees over lanes and
waves), so a sum of terms t_i is off by at most c u sum |t_i|; what is computed
from it adds a few roundings more, for which c has room.  A result stored as
bfloat16 is rounded once, 2^-8 of its value at most.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"


@pytest.fixture(scope="module")
def tc():
    import paper_1801_03855_amd as tc
    tc.lib()
    return tc


def chain(cols):
    return (64 + cols / 128) * U


def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def rows_of(gen, rows, cols, pad, dtype, scale=1.0, shift=0.0):
    t = torch.randn(rows, cols + pad, generator=gen, dtype=torch.float64) * scale + shift
    return t.to(dtype).to(DEV)[:, :cols]


def vectors(gen, K, cols, offset, base=0.0):
    """K pieces of flat buffers that start `offset` elements into them."""
    return [(torch.randn(offset + cols + 3, generator=gen) * 0.5 + base).to(DEV)[offset:offset + cols] for _ in range(K)]


def within(got, want, bound, what):
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    bad = ((got - want).abs() > bound) & ~torch.isnan(want)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} off, worst {float(((got - want).abs() / bound)[bad].max()):.2f} of its bound"


def forward_formula(x, w, b, eps):
    x = x.double()
    n = x.shape[1]
    mean = x.sum(1, keepdim=True) / n
    var = ((x - mean) ** 2).sum(1, keepdim=True) / n
    r = 1 / torch.sqrt(var + eps)
    xh = (x - mean) * r
    return xh * w + b, mean, r, xh


def check_forward(x, w, b, y, mean, rstd, eps):
    x, w, b = x.cpu(), w.cpu().double(), b.cpu().double()
    c = chain(x.shape[1])
    want, m, r, xh = forward_formula(x, w, b, eps)
    size = x.double().abs().mean(1, keepdim=True)
    # the mean's own error moves every difference to it; the variance's error is
    # at most c of its value plus the square of that
    moved = c * size
    bound = w.abs() * r * (moved + 4 * U * (x.double().abs() + m.abs())) + (w * xh).abs() * (c + (moved * r) ** 2) + c * b.abs() * 0.1
    within(y, want, bound + half_ulp(y.dtype) * want.abs() + 1e-38, "y")
    within(mean, m[:, 0], moved[:, 0] + 1e-38, "mean")
    within(rstd, r[:, 0], r[:, 0] * (c + (moved * r)[:, 0] ** 2), "rstd")


def check_backward(dy, x, w, mean, rstd, dx, dw, db):
    dy, x, w = dy.cpu().double(), x.cpu().double(), w.cpu().double()
    m, r = mean.cpu().double()[:, None], rstd.cpu().double()[:, None]
    n, c = x.shape[1], chain(x.shape[1])
    xh = (x - m) * r
    exh = 4 * U * (x.abs() + m.abs()) * r  # of xh: the difference and a product
    h = dy * w
    along = (h * xh).sum(1, keepdim=True) / n
    want = r * (h - h.sum(1, keepdim=True) / n - xh * along)
    bound = r * (4 * U * h.abs() + c * h.abs().mean(1, keepdim=True) + (exh + 4 * U * xh.abs()) * along.abs()
                 + xh.abs() * (c * (h * xh).abs().mean(1, keepdim=True) + (h.abs() * exh).mean(1, keepdim=True)))
    within(dx, want, bound + half_ulp(dx.dtype) * want.abs() + 1e-38, "dx")
    rows = (x.shape[0] + 64) * U  # a chain over all rows at most
    want = (dy * xh).sum(0)
    within(dw, want, rows * (dy * xh).abs().sum(0) + (dy.abs() * exh).sum(0) + half_ulp(dw.dtype) * want.abs() + 1e-38, "dw")
    want = dy.sum(0)
    within(db, want, rows * dy.abs().sum(0) + half_ulp(db.dtype) * want.abs() + 1e-38, "db")


def make(gen, rows, cols, dtype, pad=0, shift=0.25, offset=0):
    K = len(rows)
    xs = [rows_of(gen, r, cols, pad, dtype, 1.5, shift) for r in rows]
    dys = [rows_of(gen, r, cols, pad, dtype, 0.1) for r in rows]
    return xs, dys, vectors(gen, K, cols, offset, 1.0), vectors(gen, K, cols, offset)


def forward(tc, xs, ws, bs, eps=1e-5, **kw):
    ys = [torch.full_like(x, 7.0) for x in xs]
    means = [torch.full((x.shape[0],), 7.0, device=DEV) for x in xs]
    rstds = [torch.full((x.shape[0],), 7.0, device=DEV) for x in xs]
    tc.layernorm(xs, ws, bs, ys, means, rstds, eps, **kw)
    return ys, means, rstds


def backward(tc, dys, xs, ws, means, rstds, w_dtype, offset=0, **kw):
    cols = xs[0].shape[1]
    dxs = [torch.full_like(x, 7.0) for x in xs]
    flat = [[torch.full((offset + cols + 2,), 7.0, dtype=w_dtype, device=DEV) for _ in xs] for _ in range(2)]
    dws, dbs = [[f[offset:offset + cols] for f in fs] for fs in flat]
    tc.layernorm_backward(dys, xs, ws, means, rstds, dxs, dws, dbs, **kw)
    for fs in flat:
        for f in fs:  # nothing outside the pieces is written
            assert float(f[offset + cols:].float().min()) == 7.0 and (offset == 0 or float(f[:offset].float().min()) == 7.0)
    return dxs, dws, dbs


# every shape of the kernels: lanes of a wave, a wave, workgroups of both
# sizes, and rows too long for registers; at, below and above their edges
COLS = [1, 2, 7, 31, 32, 33, 63, 64, 65, 129, 255, 256, 257, 300, 511, 513, 777, 1000, 1023, 1024, 1025, 2047, 2049,
        4095, 4096, 4097, 8191, 8200, 16383, 16384, 16385, 20001, 40000]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", COLS)
def test_both_passes_at_every_width(tc, cols, dtype):
    gen = torch.Generator().manual_seed(cols)
    rows = [5, 0, 18] if cols > 2000 else [37, 0, 130]
    xs, dys, ws, bs = make(gen, rows, cols, dtype, pad=cols % 3, offset=cols % 4)
    ys, means, rstds = forward(tc, xs, ws, bs)
    dxs, dws, dbs = backward(tc, dys, xs, ws, means, rstds, dtype, offset=cols % 4)
    for k, r in enumerate(rows):
        if r:
            check_forward(xs[k], ws[k], bs[k], ys[k], means[k], rstds[k], 1e-5)
        check_backward(dys[k], xs[k], ws[k], means[k], rstds[k], dxs[k], dws[k], dbs[k])


@pytest.mark.parametrize("K,rows,cols,dtype,w_dtype", [
    (1, 1, 512, torch.float32, torch.float32), (2, 1, 4096, torch.bfloat16, torch.float32),
    (33, 3, 96, torch.float32, torch.bfloat16), (64, 2, 130, torch.bfloat16, torch.bfloat16),
    (3, 2777, 256, torch.float32, torch.float32), (2, 9001, 40, torch.bfloat16, torch.bfloat16),
    (4, 700, 2048, torch.bfloat16, torch.float32), (1, 600, 16384, torch.bfloat16, torch.bfloat16),
    (2, 90, 17000, torch.float32, torch.float32),
])
def test_many_workers_and_rows(tc, K, rows, cols, dtype, w_dtype):
    gen = torch.Generator().manual_seed(K * 1000 + cols)
    counts = [max(0, rows - 3 * (k % 2)) for k in range(K)]
    xs, dys, ws, bs = make(gen, counts, cols, dtype)
    ys, means, rstds = forward(tc, xs, ws, bs)
    dxs, dws, dbs = backward(tc, dys, xs, ws, means, rstds, w_dtype)
    for k in sorted({0, 1 % K, K // 2, K - 1}):
        if counts[k]:
            check_forward(xs[k], ws[k], bs[k], ys[k], means[k], rstds[k], 1e-5)
        check_backward(dys[k], xs[k], ws[k], means[k], rstds[k], dxs[k], dws[k], dbs[k])


def test_a_large_mean_costs_no_variance(tc):
    """Rows around 1,000 with a deviation of 0.01, held exactly in binary32: a
    difference of sums of squares would have nothing left of the variance."""
    gen = torch.Generator().manual_seed(5)
    x = (1000 + (torch.randint(-160, 161, (9, 640), generator=gen).double() / 8192)).float().to(DEV)
    w, b = torch.ones(640, device=DEV), torch.zeros(640, device=DEV)
    (y,), (m,), (r,) = forward(tc, [x], [w], [b], eps=0.0)
    check_forward(x, w, b, y, m, r, 0.0)


def test_constant_rows_and_rows_that_are_not_finite(tc):
    x = torch.zeros(5, 100, device=DEV)
    x[1] = 3.0
    x[2, 99] = float("inf")
    x[3, 0] = float("nan")
    x[4] = torch.arange(100, device=DEV)
    w, b = torch.full((100,), 2.0, device=DEV), torch.full((100,), 0.5, device=DEV)
    (y,), (m,), (r,) = forward(tc, [x], [w], [b])
    assert torch.equal(y[:2].cpu(), torch.full((2, 100), 0.5))
    assert bool(torch.isnan(y[2:4]).all())  # inf - inf in every difference
    check_forward(x[4:], w, b, y[4:], m[4:], r[4:], 1e-5)
    dy = torch.ones_like(x)
    (dx,), (dw,), (db,) = backward(tc, [dy], [x], [w], [m], [r], torch.float32)
    assert bool(torch.isnan(dx[2:4]).all()) and bool(torch.isfinite(dx[:2]).all()) and bool(torch.isfinite(dx[4]).all())
    assert bool(torch.isnan(dw).all()) and torch.equal(db.cpu(), torch.full((100,), 5.0))


def test_without_scale_shift_or_statistics(tc):
    gen = torch.Generator().manual_seed(9)
    xs, dys, _, _ = make(gen, [12, 4], 200, torch.float32)
    ys = [torch.empty_like(x) for x in xs]
    tc.layernorm(xs, None, None, ys)
    one, zero = torch.ones(200, device=DEV), torch.zeros(200, device=DEV)
    full, means, rstds = forward(tc, xs, [one, one], [zero, zero])
    for a, b in zip(ys, full):
        assert torch.equal(a, b)
    with_w = backward(tc, dys, xs, [one, one], means, rstds, torch.float32)
    for a, b in zip(sum(backward(tc, dys, xs, None, means, rstds, torch.float32), []), sum(with_w, [])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("cols", [96, 2000, 16384, 18000])
def test_in_place_and_interleaved_views(tc, cols):
    gen = torch.Generator().manual_seed(cols)
    xs, dys, ws, bs = make(gen, [23, 9], cols, torch.float32)
    ys, means, rstds = forward(tc, xs, ws, bs)
    dxs, dws, dbs = backward(tc, dys, xs, ws, means, rstds, torch.float32)
    for target in ("dy", "x"):
        d, x = [t.clone() for t in dys], [t.clone() for t in xs]
        w2 = [torch.empty(cols, device=DEV) for _ in xs]
        b2 = [torch.empty(cols, device=DEV) for _ in xs]
        tc.layernorm_backward(d, x, ws, means, rstds, d if target == "dy" else x, w2, b2)
        for k in range(2):
            assert torch.equal((d if target == "dy" else x)[k], dxs[k]) and torch.equal(w2[k], dws[k]) and torch.equal(b2[k], dbs[k])
    x = [t.clone() for t in xs]
    tc.layernorm(x, ws, bs, x)
    assert all(torch.equal(a, b) for a, b in zip(x, ys))
    # input and output as the halves of one wider buffer's rows
    wide = [torch.zeros(t.shape[0], 2 * cols, device=DEV) for t in xs]
    for a, b in zip(wide, xs):
        a[:, :cols] = b
    tc.layernorm([a[:, :cols] for a in wide], ws, bs, [a[:, cols:] for a in wide])
    assert all(torch.equal(a[:, cols:], y) and torch.equal(a[:, :cols], x) for a, x, y in zip(wide, xs, ys))


def test_the_gradient_against_differences(tc):
    """The loss sum(dy * y) along random directions of x, the scale and the
    shift.  Its central difference over 2h is off by O(h^2) of the derivative
    and by the forward's rounding, about 64 u sum|dy| |y| / h: with h = 0.02,
    values around 1 and 192 elements, under 2e-3 of |gradient| |direction|."""
    gen = torch.Generator().manual_seed(11)
    (x,), (dy,), (w,), (b,) = make(gen, [3], 64, torch.float32)
    dy = dy * 10

    def loss(x, w, b):
        (y,), _, _ = forward(tc, [x], [w], [b])
        return float((y.double() * dy.double()).sum())

    _, m, r = forward(tc, [x], [w], [b])
    (dx,), (dw,), (db,) = backward(tc, [dy], [x], [w], m, r, torch.float32)
    h = 0.02
    for i, g in enumerate((dx, dw, db)):
        for s in range(4):
            v = torch.randn(g.shape, generator=torch.Generator().manual_seed(100 * i + s)).to(DEV)
            at = [[x, w, b], [x, w, b]]
            at[0][i], at[1][i] = at[0][i] + h * v, at[1][i] - h * v
            slope = (loss(*at[0]) - loss(*at[1])) / (2 * h)
            want = float((g.double() * v.double()).sum())
            assert abs(slope - want) <= 2e-3 * float(g.double().norm() * v.double().norm()), (i, s)


def test_same_bits_again_and_on_another_stream(tc):
    gen = torch.Generator().manual_seed(21)
    xs, dys, ws, bs = make(gen, [900, 777], 1030, torch.bfloat16)
    first = forward(tc, xs, ws, bs)
    grads = backward(tc, dys, xs, ws, first[1], first[2], torch.float32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [[torch.empty_like(t) for t in ts] for ts in (*first, *grads)]
    side.wait_stream(torch.cuda.current_stream())
    tc.layernorm(xs, ws, bs, outs[0], outs[1], outs[2], stream=side)
    tc.layernorm_backward(dys, xs, ws, outs[1], outs[2], outs[3], outs[4], outs[5], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(sum(outs, []), sum((*first, *grads), [])):
        assert torch.equal(a, b)


def test_replayed_from_a_graph(tc):
    gen = torch.Generator().manual_seed(31)
    xs, dys, ws, bs = make(gen, [130, 70], 520, torch.float32)
    ys = [torch.empty_like(x) for x in xs]
    means, rstds = [[torch.empty(x.shape[0], device=DEV) for x in xs] for _ in range(2)]
    dxs = [torch.empty_like(x) for x in xs]
    dws, dbs = [[torch.empty(520, device=DEV) for _ in xs] for _ in range(2)]
    space = torch.empty(tc.layernorm_workspace([130, 70], 520), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tc.layernorm(xs, ws, bs, ys, means, rstds)
        tc.layernorm_backward(dys, xs, ws, means, rstds, dxs, dws, dbs, space)
    for turn in range(3):
        for x in xs:
            x.add_(0.25 * turn).mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        want = forward(tc, xs, ws, bs)
        grads = backward(tc, dys, xs, ws, want[1], want[2], torch.float32)
        for a, b in zip(sum((ys, means, rstds, dxs, dws, dbs), []), sum((*want, *grads), [])):
            assert torch.equal(a, b), turn


def test_rows_past_two_to_the_31_elements(tc):
    """Offsets of rows that do not fit 32 bits: a row stride of 2^22 elements
    (nearly all of it padding) over 600 rows, 2.5e9 elements of bfloat16."""
    rows, cols, ld = 600, 64, 1 << 22
    buf = torch.zeros(rows * ld, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (rows, cols), (ld, 1))
    x.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16))
    w, b = torch.ones(cols, device=DEV), torch.zeros(cols, device=DEV)
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    m, r = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    tc.layernorm([x], [w], [b], [y], [m], [r])
    check_forward(x, w, b, y, m, r, 1e-5)
    dx, dw, db = torch.empty_like(y), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    tc.layernorm_backward([y], [x], [w], [m], [r], [dx], [dw], [db])
    check_backward(y, x, w, m, r, dx, dw, db)


def test_refusals(tc):
    x = torch.zeros(4, 32, device=DEV)
    y, w = torch.zeros_like(x), torch.ones(32, device=DEV)
    m, r = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    dw, db = torch.zeros(32, device=DEV), torch.zeros(32, device=DEV)

    def refused(kind, fn, *a, **kw):
        with pytest.raises(kind):
            fn(*a, **kw)

    refused(ValueError, tc.layernorm, [], None, None, [])
    refused(ValueError, tc.layernorm, [x.view(-1)], None, None, [y])
    refused(TypeError, tc.layernorm, [x.half()], None, None, [y.half()])
    refused(TypeError, tc.layernorm, [x], None, None, [y.bfloat16()])
    refused(ValueError, tc.layernorm, [x], None, None, [y[:3]])
    refused(ValueError, tc.layernorm, [x], None, None, [torch.zeros(32, 4, device=DEV).t()])
    refused(ValueError, tc.layernorm, [x], [w[:31]], None, [y])
    refused(TypeError, tc.layernorm, [x], [w.bfloat16()], None, [y])
    refused(ValueError, tc.layernorm, [x], [w, w], None, [y])
    refused(ValueError, tc.layernorm, [x, torch.zeros(4, 64, device=DEV)[:, :32]], None, None, [y, y.clone()])
    refused(tc.TCError, tc.layernorm, [x[:1].expand(4, 32)], None, None, [y])
    refused(tc.TCError, tc.layernorm, [x], None, None, [y], eps=-1.0)
    refused(tc.TCError, tc.layernorm, [x], None, None, [y], eps=float("nan"))
    refused(tc.TCError, tc.layernorm, [x[:3]], None, None, [x[1:]])
    refused(tc.TCError, tc.layernorm, [x, x.clone()], None, None, [y, y])
    refused(tc.TCError, tc.layernorm, [x] * 65, None, None, [y] * 65)
    refused(tc.TCError, tc.layernorm, [torch.zeros(4, 0, device=DEV)], None, None, [torch.zeros(4, 0, device=DEV)])
    refused(tc.TCError, tc.layernorm_workspace, [4], 0)
    refused(tc.TCError, tc.layernorm_workspace, [-1], 8)
    args = [[y], [x], [w], [m], [r], [torch.zeros_like(x)], [dw], [db]]

    def back(**change):
        a = list(args)
        for i, v in change.items():
            a[int(i[1:])] = v
        return a

    refused(tc.TCError, tc.layernorm_backward, *back(_7=[dw]))
    refused(tc.TCError, tc.layernorm_backward, *back(_2=[dw]))
    refused(tc.TCError, tc.layernorm_backward, *back(_6=[y.view(-1)[:32]]))
    refused(tc.TCError, tc.layernorm_backward, *back(), workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    refused(ValueError, tc.layernorm_backward, *back(_3=[m[:3]]))
    refused(TypeError, tc.layernorm_backward, *back(_7=[db.bfloat16()]))
    refused(ValueError, tc.layernorm_backward, *back(), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    assert float(y.abs().max()) == 0.0 and float(dw.abs().max()) == 0.0
    tc.layernorm_backward(*args)
    tc.layernorm([torch.zeros(0, 8, device=DEV)], None, None, [torch.zeros(0, 8, device=DEV)])
    tc.layernorm_backward([x[:0]], [x[:0]], None, [m[:0]], [r[:0]], [x[:0]], [dw.fill_(3.0)], [db.fill_(3.0)])
    assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0


def test_abi_refuses_null_arrays(tc):
    import ctypes
    L = tc.lib()
    rows = (ctypes.c_int64 * 1)(2)
    p = (ctypes.c_void_p * 1)()
    assert L.tc_layernorm(1, None, 8, p, 8, 0, None, None, p, 8, None, None, 1e-5, None) == tc.TC_EINVAL
    assert L.tc_layernorm(1, rows, 8, None, 8, 0, None, None, p, 8, None, None, 1e-5, None) == tc.TC_EINVAL
    assert L.tc_layernorm(1, rows, 8, p, 8, 0, None, None, p, 8, None, None, 1e-5, None) == tc.TC_EINVAL
    assert L.tc_layernorm(1, rows, 8, p, 7, 0, None, None, p, 8, None, None, 1e-5, None) == tc.TC_EINVAL
    assert L.tc_layernorm(1, rows, 8, p, 8, 3, None, None, p, 8, None, None, 1e-5, None) == tc.TC_EINVAL
    assert L.tc_layernorm_workspace(1, None, 8) == -1
    assert L.tc_layernorm_backward(1, rows, 8, p, 8, p, 8, 0, None, None, None, p, 8, None, None, 0, None, 0, None) == tc.TC_EINVAL


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("base", [8, 24, 64, 1016, 1024, 4096, 8192, 12280, 12288])
def test_every_remainder_of_a_vector(tc, base, dtype):
    """Rows that end 0 to 7 elements into a 16-byte vector, in place, in views
    whose columns past the row's end are NaN and stay as they are."""
    gen = torch.Generator().manual_seed(base)
    for cols in range(base, base + 8):
        rows = [5, 0, 9]
        wide = [[torch.full((r, cols + 9), float("nan"), dtype=dtype, device=DEV) for r in rows] for _ in range(2)]
        xs, dys, ws, bs = make(gen, rows, cols, dtype, 0, offset=cols % 3)
        vx, vd = [[t[:, 1:cols + 1] for t in ts] for ts in wide]
        for v, t in zip(vx + vd, xs + dys):
            v.copy_(t)
        means = [torch.empty(r, device=DEV) for r in rows]
        rstds = [torch.empty(r, device=DEV) for r in rows]
        tc.layernorm(vx, ws, bs, vx, means, rstds)
        for k, x in enumerate(xs):
            check_forward(x, ws[k], bs[k], vx[k], means[k], rstds[k], 1e-5)
            vx[k].copy_(x)
        dws, dbs = [[torch.empty(cols, device=DEV) for _ in rows] for _ in range(2)]
        tc.layernorm_backward(vd, vx, ws, means, rstds, vd, dws, dbs)
        for k, x in enumerate(xs):
            check_backward(dys[k], x, ws[k], means[k], rstds[k], vd[k], dws[k], dbs[k])
        for ts in wide:
            for t in ts:
                assert bool(torch.isnan(t[:, 0]).all()) and bool(torch.isnan(t[:, cols + 1:]).all())
