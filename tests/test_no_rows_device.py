"""Gradients of workers that all have no rows are zeros, written where their
parameters are: on another device than the current one they are refused, as rows
are.  On the CPU, over a runtime that only says where things are."""

import shutil
import subprocess
import sys

import pytest
import torch

import paper_1801_03855_amd as tc
from paper_1801_03855_amd import build as b
from tests.test_norm_device import RUNTIME

pytestmark = [pytest.mark.skipif(torch.cuda.device_count() > 0, reason="a runtime that only says where things are"),
              pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")]

CALL = r"""
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
L.tc_last_error.restype = ctypes.c_char_p
base, n = int(sys.argv[3], 0), None
rows = (ctypes.c_int64 * 2)(0, 0)
none = (ctypes.c_void_p * 2)(None, None)
def p(at):
    return (ctypes.c_void_p * 2)(base + at, base + at + 0x10000)
i, l, f = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
ws = ctypes.c_void_p(base + 0x1000000)
status = L.tc_layernorm_backward(i(2), rows, l(64), none, l(64), none, l(64), i(0), n, none, none, none, l(64), p(0), p(0x20000), i(0), ws, l(1 << 24), n)
print(status, L.tc_last_error().decode())
status = L.tc_cross_entropy_backward(i(2), rows, l(64), l(100), none, l(64), i(0), none, n, i(0), none, none, n, f(1.0), none, l(64), p(0), p(0x20000), i(0),
                                     ws, l(1 << 24), n)
print(status, L.tc_last_error().decode())
"""


def test_gradients_of_no_rows_on_a_device_that_is_not_current(tmp_path):
    (tmp_path / "runtime.cpp").write_text(RUNTIME)
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(tmp_path / "runtime.so"), str(tmp_path / "runtime.cpp")], check=True)

    def statuses(base):
        out = subprocess.run([sys.executable, "-c", CALL, str(tmp_path / "runtime.so"), b.LIBRARY, hex(base)], check=True, capture_output=True, text=True)
        return out.stdout.splitlines()

    lines = statuses(0x1000000)
    assert len(lines) == 2
    for line in lines:
        assert line == f"{tc.TC_EINVAL} dweight[0] is on device 0 but device 1 is current"
    for line in statuses(0x1_0000_0000):  # the current one: on to the launch, for which there is no device
        assert int(line.split()[0]) not in (0, tc.TC_EINVAL), line
