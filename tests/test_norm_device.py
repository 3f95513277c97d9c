"""Layer norm with tensors on a device that is not the current one, or on two,
is refused, as every call on a group is.  On the CPU: tensors and a runtime that
only say where things are."""

import ctypes
import shutil
import subprocess
import sys

import pytest
import torch

import paper_1801_03855_amd as tc
from paper_1801_03855_amd import build as b

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="a runtime that only says where things are")


class Rows:
    """What the calls ask of a tensor."""

    is_cuda = True

    def __init__(self, device, *shape):
        self.device, self.shape, self.dtype = torch.device("cuda", device), torch.Size(shape), torch.float32
        self.at = 0x100000 + id(self) % 0x10000 * 0x10000

    def get_device(self):
        return self.device.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return (self.shape[-1], 1)

    def is_contiguous(self):
        return True

    def element_size(self):
        return 4

    def data_ptr(self):
        return self.at


@pytest.fixture
def recorded(monkeypatch):
    """The calls that reach the library."""
    calls = []

    class Library:
        def tc_layernorm(self, *a):
            calls.append("forward")
            return 0

        def tc_layernorm_backward(self, *a):
            calls.append("backward")
            return 0

        def tc_layernorm_workspace(self, *a):
            return 4096

    monkeypatch.setattr(tc, "lib", lambda: Library())
    monkeypatch.setattr(tc, "_stream", lambda stream: 0)
    return calls


def forward(**on):
    where = {n: on.get(n, 0) for n in ("x", "w", "b", "y", "mean", "rstd")}
    x, y = [[Rows(0, 4, 64), Rows(where[n], 4, 64)] for n in ("x", "y")]
    w, bias = [[Rows(0, 64), Rows(where[n], 64)] for n in ("w", "b")]
    mean, rstd = [[Rows(0, 4), Rows(where[n], 4)] for n in ("mean", "rstd")]
    tc.layernorm(x, w, bias, y, mean, rstd)


def backward(**on):
    where = {n: on.get(n, 0) for n in ("dy", "x", "w", "mean", "rstd", "dx", "dw", "db", "workspace")}
    dy, x, dx = [[Rows(0, 4, 64), Rows(where[n], 4, 64)] for n in ("dy", "x", "dx")]
    w, dw, db = [[Rows(0, 64), Rows(where[n], 64)] for n in ("w", "dw", "db")]
    mean, rstd = [[Rows(0, 4), Rows(where[n], 4)] for n in ("mean", "rstd")]
    tc.layernorm_backward(dy, x, w, mean, rstd, dx, dw, db, Rows(where["workspace"], 1024))


@pytest.mark.parametrize("call,name", [(forward, n) for n in ("x", "w", "b", "y", "mean", "rstd")]
                         + [(backward, n) for n in ("dy", "x", "w", "mean", "rstd", "dx", "dw", "db", "workspace")])
def test_one_tensor_on_another_device(recorded, call, name):
    call()
    assert recorded == [call.__name__]
    with pytest.raises(ValueError):
        call(**{name: 1})
    assert recorded == [call.__name__]


RUNTIME = r"""
#include <cstring>
extern "C" {
int hipGetDevice(int* d) { *d = 1; return 0; }
// type (2: device memory), device
int hipPointerGetAttributes(void* a, const void* p) {
    int v[2] = {2, reinterpret_cast<unsigned long>(p) >> 32 ? 1 : 0};
    memcpy(a, v, sizeof v);
    return 0;
}
}
"""
CALL = r"""
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
L.tc_last_error.restype = ctypes.c_char_p
base = int(sys.argv[3], 0)
rows = (ctypes.c_int64 * 2)(0, 4)
def p(at):
    return (ctypes.c_void_p * 2)(None, base + at)
i, l, f, n = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, None
w = (ctypes.c_void_p * 2)(base + 0x50000, base + 0x60000)
for status in (L.tc_layernorm(i(2), rows, l(64), p(0), l(64), i(0), n, n, p(0x10000), l(64), n, n, f(1e-5), n),
               L.tc_layernorm_backward(i(2), rows, l(64), p(0), l(64), p(0x10000), l(64), i(0), n, p(0x20000), p(0x30000), p(0x40000), l(64),
                                       w, (ctypes.c_void_p * 2)(base + 0x70000, base + 0x80000), i(0), ctypes.c_void_p(base + 0x100000),
                                       l(1 << 20), n)):
    print(status, L.tc_last_error().decode())
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_rows_of_a_device_that_is_not_current(tmp_path):
    (tmp_path / "runtime.cpp").write_text(RUNTIME)
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(tmp_path / "runtime.so"), str(tmp_path / "runtime.cpp")], check=True)

    def statuses(base):
        out = subprocess.run([sys.executable, "-c", CALL, str(tmp_path / "runtime.so"), b.LIBRARY, hex(base)], check=True, capture_output=True, text=True)
        return out.stdout.splitlines()

    for line in statuses(0x1000000):
        assert line == f"{tc.TC_EINVAL} x[1] is on device 0 but device 1 is current"
    for line in statuses(0x1_0000_0000):  # the current one: on to the launch, for which there is no device
        assert int(line.split()[0]) not in (0, tc.TC_EINVAL), line
