"""The cross entropy's launches, on the CPU: their grids are ones that HIP takes,
up to the largest sizes that the calls accept."""

import shutil

import pytest
import torch

from tests.launches import call, launches
from tests.loss_tiles import TILES

pytestmark = [pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses"),
              pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")]

M = 1 << 20


def check(results):
    for status, error, _, made in results:
        assert status == 0, error
        for one in made:
            assert one.fits(), (one.name, one.grid, one.block)


def test_panels_of_the_largest_operands(tmp_path):
    """2^36 elements of x, of the weight, and of both."""
    sizes = [(16 * M, 4096, 300), (8 * M + 1, 8191, 65), (70, 4096, 16 * M), (66, 8191, 8 * M + 1), (256 << 10, 256 << 10, 256 << 10)]
    check(launches(tmp_path, [call("ce", [r], c, v, "bf16", "bf16") for r, c, v in sizes]))


def test_the_tiles_of_the_sizes_that_are_compared(tmp_path):
    """tests/test_gpu_loss_tiles.py compares these with 64 bits."""
    calls, want = [], []
    for rows, cols, classes, x, w, dw, forward, backward in TILES:
        calls.append(call("ce", rows, cols, classes, x, w))
        want.append({f"loss_logit_kernelILi{forward[0]}": forward[1], "loss_join_kernel": 1})
        if backward:
            logits, products, pieces = backward
            calls.append(call("ce_grad", rows, cols, classes, x, w, dw, weighted=True))
            want.append({f"loss_logit_kernelILi{logits}": pieces, f"loss_grad_kernelILi{products}": pieces, "loss_bias_kernel": pieces})
    for c, (status, error, _, made), names in zip(calls, launches(tmp_path, calls), want):
        assert status == 0, error
        for name, count in names.items():
            assert sum(name in one.name for one in made) == count, (c, name, [one.name for one in made])
