"""Dropout past the caches, and where a lane has several turns: every element
against the formula, with a mask that torch's integer operations make."""

import numpy as np
import pytest
import torch

import paper_1801_03855_amd as tc
from tests.dropout_large import LARGE
from tests.philox import keep_mask

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, STEP, SITE, P = 0x1234567890ABCDE, 0x2FEDCBA98765, 7, 0.3
T = int(np.floor(float(np.float32(P)) * 65536 + 0.5))
M32 = 0xFFFFFFFF


def halves(a, m):
    """The high and low half of a x m, of words a in 64-bit integers (products of 32 by 16 bits, which fit)."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    low = low + ((high & 0xFFFF) << 16)
    return (high >> 16) + (low >> 32), low & M32


def keep_on_gpu(worker, rows, cols):
    per = -(-cols // 8)
    q = torch.arange(rows * per, device="cuda")
    c = [q & M32, (q >> 32) + (worker << 16), torch.full_like(q, STEP & M32), torch.full_like(q, (STEP >> 32 & 0xFFFF) << 16 | SITE)]
    k0, k1 = SEED & M32, SEED >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = halves(c[0], 0xD2511F53), halves(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    u = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], 1)
    return u.view(rows, per * 8)[:, :cols] >= T


def test_the_mask_is_the_same_as_numpy_makes():
    for worker, rows, cols in ((0, 5, 16), (3, 40, 1003)):
        assert np.array_equal(keep_on_gpu(worker, rows, cols).cpu().numpy(), keep_mask(SEED, STEP, worker, SITE, rows, cols, T))


def view(rows, cols, pad, dtype, gen):
    wide = torch.randn(rows, cols + pad, generator=gen, device="cuda").to(dtype)
    return wide, wide[:, :cols]


@pytest.mark.parametrize("place", ["y", "x", "residual"])
@pytest.mark.parametrize("rows,cols,dtype,residual,pad,past", LARGE, ids=str)
def test_every_element(rows, cols, dtype, residual, pad, past, place):
    if place == "residual" and not residual:
        place = "y"
    dtype, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(3)
    x, r, y = [[view(n, cols, pad, dtype, gen) for n in rows] for _ in range(3)]
    out = {"x": x, "residual": r, "y": y}[place]
    behind = [w[:, cols:].clone() for w, _ in out]
    half = torch.finfo(dtype).eps / 2
    expected = []
    for k, n in enumerate(rows):
        want = torch.where(keep_on_gpu(k, n, cols), x[k][1].double() * (65536 / (65536 - T)), 0.0)
        size = want.abs()
        if residual:
            want = want + r[k][1].double()
        # the product and the sum in binary32, rounded once
        expected.append((want, want.abs() * (half + 2.0 ** -24) + size * 2.0 ** -22))
    random = torch.tensor([SEED, STEP], dtype=torch.int64, device="cuda")
    tc.dropout([t for _, t in x], [t for _, t in r] if residual else None, [t for _, t in out], random, site=SITE, p=P)
    torch.cuda.synchronize()
    for (want, off), (wide, got), rest in zip(expected, out, behind):
        assert bool(((got.double() - want).abs() <= off).all())
        assert torch.equal(wide[:, cols:], rest)


@pytest.mark.parametrize("rows,cols,dtype,residual,pad,past", [c for c in LARGE if not c[3]], ids=str)
def test_the_gradient(rows, cols, dtype, residual, pad, past):
    """The backward call of ones is the mask times its factor."""
    dtype = TYPES[dtype]
    dys = [torch.ones(n, cols + pad, dtype=dtype, device="cuda")[:, :cols] for n in rows]
    dxs = [torch.full((n, cols + pad), 7.0, dtype=dtype, device="cuda")[:, :cols] for n in rows]
    tc.dropout_backward(dys, dxs, torch.tensor([SEED, STEP], dtype=torch.int64, device="cuda"), site=SITE, p=P)
    torch.cuda.synchronize()
    factor = torch.tensor(65536 / (65536 - T)).to(dtype)
    for k, (n, dx) in enumerate(zip(rows, dxs)):
        assert torch.equal(dx, torch.where(keep_on_gpu(k, n, cols), factor.to("cuda"), 0.0).to(dtype))
