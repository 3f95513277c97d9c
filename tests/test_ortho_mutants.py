"""That a comparison with a binary32 iteration shows a product of the
orthogonalised update which has lost half of an operand: the iteration with one
operand of one kind of product rounded to a single binary16 value, on the CPU."""

import pytest
import torch

A, B, C = 3.4445, -4.7750, 2.0315


def iterate(u, dtype, places=()):
    def half(name, v):
        return (v * 1024).to(torch.float16).to(dtype) / 1024 if name in places else v

    x = u.to(dtype)
    x = x / x.norm()
    for _ in range(5):
        g = half("X of X X^T", x) @ half("X of X X^T", x).t()
        p = B * g + C * (half("A", g) @ half("A", g))
        x = A * x + half("P", p) @ half("X of P X", x)
    return x


@pytest.mark.parametrize("place", ["X of X X^T", "A", "P", "X of P X"])
@pytest.mark.parametrize("shape", [(65, 65), (256, 512), (600, 1300)])
def test_a_lost_half_is_far_over_the_limit(shape, place):
    gen = torch.Generator().manual_seed(sum(shape))
    k = 1 + shape[0] // 8
    u = torch.randn(shape, generator=gen) * 0.004
    u += torch.randn(shape[0], k, generator=gen) @ torch.randn(k, shape[1], generator=gen) * (0.01 / k ** 0.5)
    want = iterate(u, torch.float64)
    plain, lost = [float((iterate(u, torch.float32, p).double() - want).norm() / want.norm()) for p in ((), (place,))]
    assert lost > 20 * plain  # the limit is 1.2
