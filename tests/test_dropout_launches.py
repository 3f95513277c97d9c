"""The kernels that dropout's large sizes take, and its grids at the limits of
the sizes; on the CPU."""

import shutil

import pytest
import torch

from tests.dropout_large import LARGE
from tests.launches import call, launches

pytestmark = [pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses"),
              pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")]


def test_the_kernels_of_the_sizes_that_are_compared(tmp_path):
    """tests/test_gpu_dropout_large.py compares these with the formula."""
    sizes = [call("dropout", rows, cols, x=x, residual=residual, pad=pad) for rows, cols, x, residual, pad, _ in LARGE]
    for (rows, cols, x, residual, _, past), (status, error, _, made) in zip(LARGE, launches(tmp_path, sizes)):
        assert status == 0, error
        (one,) = made
        kinds = (int(residual), int(cols % 8 != 0), int(past))
        assert f"dropout_kernelI{'f' if x == 'f32' else 'DF16b'}" + "".join(f"Lb{v}E" for v in kinds) in one.name
        assert sum(rows) * ((cols + 7) // 8) > 2 * one.grid[0] * one.block[0]  # more than one turn


def test_grids_up_to_the_limits(tmp_path):
    sizes = [([1 << 48], 1), ([1 << 24], 1 << 24), ([1 << 30] * 64, 1 << 18), ([1] * 64, 1), ([1] * 64, 1 << 24)]
    results = launches(tmp_path, [call("dropout", rows, cols, x=x, residual=r) for rows, cols in sizes for x in ("f32", "bf16") for r in (False, True)])
    for status, error, _, made in results:
        assert status == 0, error
        for one in made:
            assert one.fits(), (one.name, one.grid, one.block)
