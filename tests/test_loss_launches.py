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


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_grids_up_to_the_limits(tmp_path, x):
    """Both passes at the corners of what the calls accept: many rows, classes and columns, and few of each."""
    sizes = [(M, 64, M // 4), (16 * M, 1, 16 * M), (16 * M, 4096, 300), (16 * M, 4096, 64), (64, 4096, 16 * M), (70, 4096, 16 * M), (5 * M, 200, 3 * M),
             (256 << 10, 256 << 10, 256 << 10), (16 * M, 3, 5), (3, 5, 16 * M), (1, 1, 1)]
    check(launches(tmp_path, [call(op, [r], c, v, x, x, x) for r, c, v in sizes for op in ("ce", "ce_grad")]))
    check(launches(tmp_path, [call("ce", [200] * 64, 64, M, x, x), call("ce_grad", [200] * 64, 64, M, x, x)]))


@pytest.mark.parametrize("rows,cols", [(M, 64), (16 * M, 1), (70000, 72)])
def test_the_forward_workspace_does_not_grow_with_the_classes(tmp_path, rows, cols):
    """A worker's rows as they are laid out, 256 MiB of pairs, 256 MiB of the weight's panels, and a few words a row."""
    needs = [r[2] for r in launches(tmp_path, [call("ce", [rows], cols, v, "bf16", "bf16") for v in (4 * M, 16 * M)])]
    laid_out = (rows + 255) // 256 * 256 * ((cols + 63) // 64 * 64) * 2
    assert max(needs) <= laid_out + (512 << 20) + rows * 32 + (1 << 20)


def test_how_often_pairs_are_joined(tmp_path):
    """The sizes of tests/test_gpu_loss_tiles.py, and a large one that has room for all of them."""
    sizes = [((1 << 20) - 5, 67, 9001, "bf16", 3), (1 << 20, 64, 8200, "f32", 3), (131000, 4090, 50001, "bf16", 2), (8192, 4096, 131072, "bf16", 1)]
    for (*_, joins), (status, error, _, made) in zip(sizes, launches(tmp_path, [call("ce", [r], c, v, x, x) for r, c, v, x, _ in sizes])):
        assert status == 0, error
        assert sum("loss_join_kernel" in one.name for one in made) == joins
