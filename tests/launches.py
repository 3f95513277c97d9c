"""What a call of the library launches, without a GPU: the built library in a
process of its own, over a runtime that only writes down kernels and grids.
Addresses are made up; nothing is read or written behind them."""

import json
import subprocess
import sys

from paper_1801_03855_amd import build as b

RUNTIME = r"""
#include <cstdint>
#include <cstring>
#include <map>
#include <string>

struct Dim {
    uint32_t x, y, z;
};
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static std::string text;
static Dim grid_, block_;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* p; return &p; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
int __hipPushCallConfiguration(Dim g, Dim b, size_t, void*) { grid_ = g; block_ = b; return 0; }
int __hipPopCallConfiguration(Dim* g, Dim* b, size_t* n, void** s) { *g = grid_; *b = block_; *n = 0; *s = nullptr; return 0; }
int hipLaunchKernel(const void* f, Dim g, Dim b, void**, size_t, void*) {
    text += names()[f];
    for (uint32_t v : {g.x, g.y, g.z, b.x, b.y, b.z}) text += ' ' + std::to_string(v);
    text += '\n';
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipPointerGetAttributes(void* a, const void*) {
    const int v[2] = {2, 0};  // device memory, of device 0
    memcpy(a, v, sizeof v);
    return 0;
}
void start() { text.clear(); }
const char* launched() { return text.c_str(); }
}
"""

CHILD = r"""
import ctypes, json, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
runtime.launched.restype = ctypes.c_char_p
L = ctypes.CDLL(sys.argv[2])
L.tc_last_error.restype = ctypes.c_char_p
for n in ("tc_cross_entropy_workspace", "tc_cross_entropy_backward_workspace"):
    getattr(L, n).restype = ctypes.c_int64
l, i, f, p = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p
for call in json.load(sys.stdin):
    rows, cols, K = call["rows"], call["cols"], len(call["rows"])
    counts = (ctypes.c_int64 * K)(*rows)
    at = iter(range(1, 1 << 20))
    each = lambda: (ctypes.c_void_p * K)(*[next(at) << (52 if call["op"] == "dropout" else 40) for _ in rows])
    types = ("f32", "bf16")
    x, w, dw = [i(types.index(call[n])) for n in ("x", "w", "dw")]
    if call["op"] in ("ce", "ce_grad"):
        head = (i(K), counts, l(cols), l(call["classes"]))
        bias = each() if call["bias"] else None
        if call["op"] == "ce":
            need = L.tc_cross_entropy_workspace(*head, x, w)
            args = (*head, each(), l(cols), x, each(), bias, w, each(), each(), each(), p(1 << 60), l(need), None)
            status = lambda: L.tc_cross_entropy(*args)
        else:
            need = L.tc_cross_entropy_backward_workspace(*head, x, w, dw)
            dbias, dloss = each() if call["bias"] else None, each() if call["weighted"] else None
            args = (*head, each(), l(cols), x, each(), bias, w, each(), each(), dloss, f(1.0), each(), l(cols), each(), dbias, dw, p(1 << 60), l(need), None)
            status = lambda: L.tc_cross_entropy_backward(*args)
    else:
        need = 0
        residual = each() if call["residual"] else None
        ld = l(cols + call["pad"])
        args = (i(K), counts, l(cols), each(), ld, x, residual, ld, each(), ld, f(0.5), p(1 << 60), l(0), None)
        status = lambda: L.tc_dropout(*args)
    runtime.start()
    code = status()
    print(json.dumps([code, L.tc_last_error().decode(), need, runtime.launched().decode()]))
"""


class Launch:
    def __init__(self, line):
        name, *n = line.split()
        self.name, n = name, [int(v) for v in n]
        self.grid, self.block = n[:3], n[3:]

    def fits(self):
        """HIP takes fewer than 2^32 threads in a dimension, and 65,535 workgroups along y and z."""
        return all(0 < g and g * t < 1 << 32 for g, t in zip(self.grid, self.block)) and max(self.grid[1:]) <= 65535


def call(op, rows, cols, classes=0, x="f32", w="f32", dw="f32", bias=True, weighted=False, residual=False, pad=0):
    return {"op": op, "rows": list(rows), "cols": cols, "classes": classes, "x": x, "w": w, "dw": dw, "bias": bias, "weighted": weighted,
            "residual": residual, "pad": pad}


def launches(tmp_path, calls):
    """Of every call: (status, error, workspace, launches)."""
    (tmp_path / "runtime.cpp").write_text(RUNTIME)
    runtime = str(tmp_path / "runtime.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", runtime, str(tmp_path / "runtime.cpp")], check=True)
    out = subprocess.run([sys.executable, "-c", CHILD, runtime, b.LIBRARY], input=json.dumps(calls), check=True, capture_output=True, text=True)
    results = []
    for line in out.stdout.splitlines():
        status, error, need, text = json.loads(line)
        results.append((status, error, need, [Launch(v) for v in text.splitlines()]))
    assert len(results) == len(calls)
    return results
