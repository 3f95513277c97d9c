"""Tensor-group collectives and the fused elastic-averaging SGD step on
AMD MI355X (gfx950).

A thin ctypes binding of the C ABI declared in ``include/tc.h``: every
function here marshals torch tensors into device pointers, sizes and the
current HIP stream, and calls the library of the same name.  All arithmetic
runs in the library's HIP kernels; there is no CPU or PyTorch fallback, and
loading fails loudly when the library has not been built.

    g = Group(sizes)                        # tc_group_create
    tl = TensorList(g, [[t00, t01, ...], [t10, ...]])   # tc_tensorlist_create
    pack(tl, flats); unpack(tl, flats)      # tc_pack / tc_unpack
    reduce(g, ins, out, "avg")              # tc_reduce / tc_reduce_ex
    easgd_step(g, xs, gs, xc, eta, rho)     # easgd_step / easgd_step_ex

Schedules and synchronous SGD (separate buffers; *_tensor on the tensor layout):
    sgd_step(g, xs, gs, eta)                # sgd_step
    easgd_period_step(g, xs, gs, xc, eta, rho, t, tau)  # easgd_period_step
    elastic_async(g, xs, xc, order, alpha)  # elastic_async
    sync_sgd_step(g, xs, gs, eta, rescale, broadcast)   # sync_sgd_step
    broadcast(g, src, dsts)                 # tc_broadcast

Tensor layout (the K copies interleaved in one buffer):
    n = tensor_numel(g, K)                  # tc_tensor_numel
    pack_tensor(tl, T); unpack_tensor(tl, T)            # tc_pack_tensor / tc_unpack_tensor
    reduce_tensor(g, K, T, out, "avg")      # tc_reduce_tensor
    easgd_step_tensor(g, K, X, G, xc, eta, rho)         # easgd_step_tensor

What makes the gradients and the updates:
    layernorm(xs, ws, bs, ys, means, rstds)             # tc_layernorm
    layernorm_backward(dys, xs, ws, means, rstds, dxs, dws, dbs)   # tc_layernorm_backward
    plan = OrthoPlan(g, K, shapes)                      # tc_ortho_create
    orthogonalize(plan, gs, outs, momenta)              # tc_orthogonalize
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

from .build import LIBRARY

TC_SUM, TC_AVG = 0, 1
TC_F32, TC_BF16 = 0, 1
TC_OK, TC_EINVAL, TC_ENOMEM, TC_EHIP, TC_EUNSUPPORTED = 0, -1, -2, -3, -4
TC_MAX_K = 64

_OPS = {"sum": TC_SUM, "avg": TC_AVG, TC_SUM: TC_SUM, TC_AVG: TC_AVG}
_DTYPES = {torch.float32: TC_F32, torch.bfloat16: TC_BF16}


class TCError(RuntimeError):
    """A C-ABI call returned an error status."""

    def __init__(self, status: int, message: str):
        super().__init__(f"[{status}] {message}")
        self.status = status


_VP = ctypes.c_void_p
_VPP = ctypes.POINTER(ctypes.c_void_p)
_lib = None


def lib(path: str = LIBRARY) -> ctypes.CDLL:
    """The loaded HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"HIP library {path} is not built; run __graft_entry__.build() "
                           f"or python -m paper_1801_03855_amd.build")
    L = ctypes.CDLL(path)
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    sig = {
        "tc_last_error": (ctypes.c_char_p, []),
        "tc_version": (i32, []),
        "tc_group_create": (_VP, [ctypes.POINTER(i64), i32]),
        "tc_group_destroy": (None, [_VP]),
        "tc_group_numel": (i64, [_VP]),
        "tc_group_ntensors": (i32, [_VP]),
        "tc_group_offsets": (i32, [_VP, ctypes.POINTER(i64)]),
        "tc_tensorlist_create": (_VP, [_VP, i32, _VPP, i32]),
        "tc_tensorlist_destroy": (None, [_VP]),
        "tc_pack": (i32, [_VP, _VPP, _VP]),
        "tc_unpack": (i32, [_VP, _VPP, _VP]),
        "tc_reduce": (i32, [_VP, i32, _VPP, _VP, i32, _VP]),
        "tc_reduce_ex": (i32, [_VP, i32, _VPP, i32, _VP, i32, _VP]),
        "easgd_step": (i32, [_VP, i32, _VPP, _VPP, _VP, f32, f32, _VP]),
        "easgd_step_ex": (i32, [_VP, i32, _VPP, _VPP, i32, _VP, f32, f32, _VP]),
        "reduce_easgd_step": (i32, [_VP, i32, _VPP, _VPP, i32, _VP, _VP, i32, f32, f32, _VP]),
        "tc_tensor_numel": (i64, [_VP, i32]),
        "tc_pack_tensor": (i32, [_VP, _VP, _VP]),
        "tc_unpack_tensor": (i32, [_VP, _VP, _VP]),
        "tc_reduce_tensor": (i32, [_VP, i32, _VP, i32, _VP, i32, _VP]),
        "easgd_step_tensor": (i32, [_VP, i32, _VP, _VP, i32, _VP, f32, f32, _VP]),
        "reduce_easgd_step_tensor": (i32, [_VP, i32, _VP, _VP, i32, _VP, _VP, i32, f32, f32, _VP]),
        "sgd_step": (i32, [_VP, i32, _VPP, _VPP, i32, f32, _VP]),
        "sgd_step_tensor": (i32, [_VP, i32, _VP, _VP, i32, f32, _VP]),
        "easgd_period_step": (i32, [_VP, i32, _VPP, _VPP, i32, _VP, f32, f32, i64, i32, _VP]),
        "easgd_period_step_tensor": (i32, [_VP, i32, _VP, _VP, i32, _VP, f32, f32, i64, i32, _VP]),
        "elastic_async": (i32, [_VP, i32, _VPP, _VP, ctypes.POINTER(i32), i32, f32, _VP]),
        "elastic_async_tensor": (i32, [_VP, i32, _VP, _VP, ctypes.POINTER(i32), i32, f32, _VP]),
        "sync_sgd_step": (i32, [_VP, i32, _VPP, _VPP, i32, f32, f32, i32, _VP]),
        "sync_sgd_step_tensor": (i32, [_VP, i32, _VP, _VP, i32, f32, f32, i32, _VP]),
        "tc_broadcast": (i32, [_VP, i32, _VP, _VPP, i32, _VP]),
        "tc_broadcast_tensor": (i32, [_VP, i32, _VP, _VP, i32, _VP]),
        "easgd_pipeline_tensor": (i32, [_VP, _VP, _VP, _VP, _VP, _VP, f32, f32, _VP]),
        "tc_layernorm": (i32, [i32, ctypes.POINTER(i64), i64, _VPP, i64, i32, _VPP, _VPP, _VPP, i64, _VPP, _VPP, f32, _VP]),
        "tc_layernorm_workspace": (i64, [i32, ctypes.POINTER(i64), i64]),
        "tc_layernorm_backward": (i32, [i32, ctypes.POINTER(i64), i64, _VPP, i64, _VPP, i64, i32, _VPP, _VPP, _VPP, _VPP,
                                        i64, _VPP, _VPP, i32, _VP, i64, _VP]),
        "tc_ortho_create": (_VP, [_VP, i32, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(f32)]),
        "tc_ortho_destroy": (None, [_VP]),
        "tc_ortho_workspace": (i64, [_VP]),
        "tc_orthogonalize": (i32, [_VP, _VPP, i32, _VPP, f32, i32, _VPP, i32, i32, ctypes.POINTER(f32), f32, _VP, i64, _VP]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def last_error() -> str:
    return lib().tc_last_error().decode()


def _check(status: int) -> None:
    if status != TC_OK:
        raise TCError(status, last_error())


def _ptr_array(ptrs: Sequence[Optional[int]]):
    return (ctypes.c_void_p * max(1, len(ptrs)))(*ptrs)


# The current stream's handle without a Stream object around it (a quarter of
# the host time of a small call), where this torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _elsewhere(t: torch.Tensor, device: Optional[int], what: str) -> ValueError:
    if not t.is_cuda:
        return ValueError(f"{what} must be a GPU tensor")
    return ValueError(f"{what} is on {t.device}, the first worker's rows are on device {device}")


def _dev_ptr(t: torch.Tensor, n: int, dtypes=(torch.float32,), what: str = "tensor", device: Optional[int] = None) -> int:
    if not t.is_cuda if device is None else t.get_device() != device:
        raise _elsewhere(t, device, what)
    if t.dtype not in dtypes:
        raise TypeError(f"{what} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{what} must be contiguous with at least {n} elements (has {t.numel()})")
    return t.data_ptr()


class Group:
    """A tensor group: n layer sizes, one flat index space of N elements."""

    def __init__(self, sizes: Sequence[int]):
        arr = (ctypes.c_int64 * len(sizes))(*[int(s) for s in sizes])
        h = lib().tc_group_create(arr, len(sizes))
        if not h:
            raise TCError(TC_EINVAL, last_error())
        self._h = h
        self.sizes = [int(s) for s in sizes]
        self.n = lib().tc_group_ntensors(h)
        self.numel = lib().tc_group_numel(h)

    @property
    def handle(self):
        return self._h

    def offsets(self):
        out = (ctypes.c_int64 * (self.n + 1))()
        _check(lib().tc_group_offsets(self._h, out))
        return list(out)

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.tc_group_destroy(h)


class TensorList:
    """K copies of a group as separate tensors: tensors[k][t] is tensor t of
    copy k (a contiguous GPU tensor of sizes[t] elements)."""

    def __init__(self, group: Group, tensors: Sequence[Sequence[torch.Tensor]]):
        K = len(tensors)
        if K < 1:
            raise ValueError("a tensor list needs at least one copy")
        dt = None
        ptrs = []
        for k, copy in enumerate(tensors):
            if len(copy) != group.n:
                raise ValueError(f"copy {k} has {len(copy)} tensors, the group has {group.n}")
            for t, (x, s) in enumerate(zip(copy, group.sizes)):
                dt = dt or x.dtype
                if x.dtype != dt or x.dtype not in _DTYPES:
                    raise TypeError(f"tensor ({k},{t}) has dtype {x.dtype}")
                if x.numel() != s:
                    raise ValueError(f"tensor ({k},{t}) has {x.numel()} elements, expected {s}")
                ptrs.append(_dev_ptr(x, s, (dt,), f"tensor ({k},{t})") if s else 0)
        self.group, self.K, self.dtype = group, K, dt
        self._keep = [list(c) for c in tensors]
        h = lib().tc_tensorlist_create(group.handle, K, _ptr_array(ptrs), _DTYPES[dt])
        if not h:
            raise TCError(TC_EINVAL, last_error())
        self._h = h

    @property
    def handle(self):
        return self._h

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.tc_tensorlist_destroy(h)


def _flat_ptrs(tl: TensorList, flats: Sequence[torch.Tensor]):
    if len(flats) != tl.K:
        raise ValueError(f"need {tl.K} flat buffers, got {len(flats)}")
    n = tl.group.numel
    return _ptr_array([_dev_ptr(f, n, (tl.dtype,), f"flat[{k}]") for k, f in enumerate(flats)])


def pack(tl: TensorList, flats: Sequence[torch.Tensor], stream=None) -> None:
    """flats[k][offsets[t] + e] = tensors[k][t][e] (tc_pack)."""
    _check(lib().tc_pack(tl.handle, _flat_ptrs(tl, flats), _stream(stream)))


def unpack(tl: TensorList, flats: Sequence[torch.Tensor], stream=None) -> None:
    """tensors[k][t][e] = flats[k][offsets[t] + e] (tc_unpack)."""
    _check(lib().tc_unpack(tl.handle, _flat_ptrs(tl, flats), _stream(stream)))


def reduce(group: Group, ins: Sequence[torch.Tensor], out: torch.Tensor, op="avg", stream=None) -> None:
    """out = sum (or average) of the K flat copies ins (tc_reduce_ex)."""
    n = group.numel
    dt = ins[0].dtype
    if dt not in _DTYPES:
        raise TypeError(f"inputs have dtype {dt}")
    p = _ptr_array([_dev_ptr(t, n, (dt,), f"in[{i}]") for i, t in enumerate(ins)])
    _check(lib().tc_reduce_ex(group.handle, len(ins), p, _DTYPES[dt],
                              _dev_ptr(out, n, (torch.float32,), "out"), _OPS[op], _stream(stream)))


def easgd_step(group: Group, xs: Sequence[torch.Tensor], gs: Sequence[torch.Tensor], xc: torch.Tensor,
               eta: float, rho: float, stream=None) -> None:
    """One fused elastic-averaging SGD step, in place on xs and xc
    (easgd_step_ex)."""
    n = group.numel
    if len(xs) != len(gs):
        raise ValueError("need one gradient per worker")
    gdt = gs[0].dtype
    if gdt not in _DTYPES:
        raise TypeError(f"gradients have dtype {gdt}")
    xp = _ptr_array([_dev_ptr(t, n, (torch.float32,), f"x[{i}]") for i, t in enumerate(xs)])
    gp = _ptr_array([_dev_ptr(t, n, (gdt,), f"grad[{i}]") for i, t in enumerate(gs)])
    _check(lib().easgd_step_ex(group.handle, len(xs), xp, gp, _DTYPES[gdt],
                               _dev_ptr(xc, n, (torch.float32,), "x_c"), float(eta), float(rho),
                               _stream(stream)))


def reduce_easgd_step(group: Group, xs: Sequence[torch.Tensor], gs: Sequence[torch.Tensor], xc: torch.Tensor,
                      out: torch.Tensor, eta: float, rho: float, op="avg", stream=None) -> None:
    """The sum (or average) of the gradients into out and the fused step on
    xs and xc, in one pass (reduce_easgd_step)."""
    n = group.numel
    if len(xs) != len(gs):
        raise ValueError("need one gradient per worker")
    gdt = gs[0].dtype
    if gdt not in _DTYPES:
        raise TypeError(f"gradients have dtype {gdt}")
    xp = _ptr_array([_dev_ptr(t, n, (torch.float32,), f"x[{i}]") for i, t in enumerate(xs)])
    gp = _ptr_array([_dev_ptr(t, n, (gdt,), f"grad[{i}]") for i, t in enumerate(gs)])
    _check(lib().reduce_easgd_step(group.handle, len(xs), xp, gp, _DTYPES[gdt],
                                   _dev_ptr(xc, n, (torch.float32,), "x_c"),
                                   _dev_ptr(out, n, (torch.float32,), "out"), _OPS[op], float(eta), float(rho),
                                   _stream(stream)))


# --------------------------------------------------------------- tensor layout

def tensor_numel(group: Group, K: int) -> int:
    n = lib().tc_tensor_numel(group.handle, K)
    if n < 0:
        raise TCError(TC_EINVAL, f"bad K = {K}")
    return n


def pack_tensor(tl: TensorList, tensor: torch.Tensor, stream=None) -> None:
    """K copies' separate tensors -> one tensor-layout buffer (tc_pack_tensor)."""
    n = tensor_numel(tl.group, tl.K)
    _check(lib().tc_pack_tensor(tl.handle, _dev_ptr(tensor, n, (tl.dtype,), "tensor"), _stream(stream)))


def unpack_tensor(tl: TensorList, tensor: torch.Tensor, stream=None) -> None:
    """One tensor-layout buffer -> the K copies' separate tensors (tc_unpack_tensor)."""
    n = tensor_numel(tl.group, tl.K)
    _check(lib().tc_unpack_tensor(tl.handle, _dev_ptr(tensor, n, (tl.dtype,), "tensor"), _stream(stream)))


def reduce_tensor(group: Group, K: int, tensor: torch.Tensor, out: torch.Tensor, op="avg", stream=None) -> None:
    """out = sum (or average) of the K copies in a tensor-layout buffer (tc_reduce_tensor)."""
    dt = tensor.dtype
    if dt not in _DTYPES:
        raise TypeError(f"input has dtype {dt}")
    p = _dev_ptr(tensor, tensor_numel(group, K), (dt,), "in")
    _check(lib().tc_reduce_tensor(group.handle, K, p, _DTYPES[dt], _dev_ptr(out, group.numel, (torch.float32,), "out"),
                                  _OPS[op], _stream(stream)))


def easgd_step_tensor(group: Group, K: int, x: torch.Tensor, g: torch.Tensor, xc: torch.Tensor,
                      eta: float, rho: float, stream=None) -> None:
    """One fused elastic-averaging SGD step on tensor-layout workers x and
    gradients g, in place on x and xc (easgd_step_tensor)."""
    n = tensor_numel(group, K)
    gdt = g.dtype
    if gdt not in _DTYPES:
        raise TypeError(f"gradients have dtype {gdt}")
    _check(lib().easgd_step_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"),
                                   _dev_ptr(g, n, (gdt,), "grad"), _DTYPES[gdt],
                                   _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), float(eta), float(rho),
                                   _stream(stream)))


def reduce_easgd_step_tensor(group: Group, K: int, x: torch.Tensor, g: torch.Tensor, xc: torch.Tensor,
                             out: torch.Tensor, eta: float, rho: float, op="avg", stream=None) -> None:
    """reduce_easgd_step on tensor-layout workers x and gradients g
    (reduce_easgd_step_tensor)."""
    n = tensor_numel(group, K)
    gdt = g.dtype
    if gdt not in _DTYPES:
        raise TypeError(f"gradients have dtype {gdt}")
    _check(lib().reduce_easgd_step_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"),
                                          _dev_ptr(g, n, (gdt,), "grad"), _DTYPES[gdt],
                                          _dev_ptr(xc, group.numel, (torch.float32,), "x_c"),
                                          _dev_ptr(out, group.numel, (torch.float32,), "out"), _OPS[op],
                                          float(eta), float(rho), _stream(stream)))


# ----------------------------------------------- schedules and synchronous SGD

def _gdt(gs_or_g) -> torch.dtype:
    dt = gs_or_g[0].dtype if isinstance(gs_or_g, (list, tuple)) else gs_or_g.dtype
    if dt not in _DTYPES:
        raise TypeError(f"gradients have dtype {dt}")
    return dt


def _workers(group: Group, xs):
    return _ptr_array([_dev_ptr(t, group.numel, (torch.float32,), f"x[{i}]") for i, t in enumerate(xs)])


def _grads(group: Group, gs, dt):
    return _ptr_array([_dev_ptr(t, group.numel, (dt,), f"grad[{i}]") for i, t in enumerate(gs)])


def sgd_step(group: Group, xs, gs, eta: float, stream=None) -> None:
    """x_i -= eta * g_i for every worker, in place (sgd_step)."""
    dt = _gdt(gs)
    _check(lib().sgd_step(group.handle, len(xs), _workers(group, xs), _grads(group, gs, dt), _DTYPES[dt],
                          float(eta), _stream(stream)))


def sgd_step_tensor(group: Group, K: int, x, g, eta: float, stream=None) -> None:
    dt = _gdt(g)
    n = tensor_numel(group, K)
    _check(lib().sgd_step_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"), _dev_ptr(g, n, (dt,), "grad"),
                                 _DTYPES[dt], float(eta), _stream(stream)))


def easgd_period_step(group: Group, xs, gs, xc, eta: float, rho: float, iteration: int, tau: int, stream=None) -> None:
    """The elastic step when iteration % tau == 0, plain SGD otherwise."""
    dt = _gdt(gs)
    _check(lib().easgd_period_step(group.handle, len(xs), _workers(group, xs), _grads(group, gs, dt), _DTYPES[dt],
                                   _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), float(eta), float(rho),
                                   int(iteration), int(tau), _stream(stream)))


def easgd_period_step_tensor(group: Group, K: int, x, g, xc, eta: float, rho: float, iteration: int, tau: int,
                             stream=None) -> None:
    dt = _gdt(g)
    n = tensor_numel(group, K)
    _check(lib().easgd_period_step_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"),
                                          _dev_ptr(g, n, (dt,), "grad"), _DTYPES[dt],
                                          _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), float(eta), float(rho),
                                          int(iteration), int(tau), _stream(stream)))


def _order(order):
    o = [int(v) for v in order]
    return (ctypes.c_int32 * max(1, len(o)))(*o), len(o)


def elastic_async(group: Group, xs, xc, order, alpha: float, stream=None) -> None:
    """Elastic exchanges of the workers in `order`, one at a time (elastic_async)."""
    arr, R = _order(order)
    _check(lib().elastic_async(group.handle, len(xs), _workers(group, xs),
                               _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), arr, R, float(alpha),
                               _stream(stream)))


def elastic_async_tensor(group: Group, K: int, x, xc, order, alpha: float, stream=None) -> None:
    arr, R = _order(order)
    n = tensor_numel(group, K)
    _check(lib().elastic_async_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"),
                                      _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), arr, R, float(alpha),
                                      _stream(stream)))


def sync_sgd_step(group: Group, xs, gs, eta: float, rescale: float, broadcast: bool = False, stream=None) -> None:
    """Synchronous SGD through pushpull (sync_sgd_step)."""
    dt = _gdt(gs)
    _check(lib().sync_sgd_step(group.handle, len(xs), _workers(group, xs), _grads(group, gs, dt), _DTYPES[dt],
                               float(eta), float(rescale), int(bool(broadcast)), _stream(stream)))


def sync_sgd_step_tensor(group: Group, K: int, x, g, eta: float, rescale: float, broadcast: bool = False,
                         stream=None) -> None:
    dt = _gdt(g)
    n = tensor_numel(group, K)
    _check(lib().sync_sgd_step_tensor(group.handle, K, _dev_ptr(x, n, (torch.float32,), "x"),
                                      _dev_ptr(g, n, (dt,), "grad"), _DTYPES[dt], float(eta), float(rescale),
                                      int(bool(broadcast)), _stream(stream)))


def broadcast(group: Group, src, dsts, stream=None) -> None:
    """dsts[i] = src for every copy (tc_broadcast)."""
    dt = _gdt(src)
    p = _ptr_array([_dev_ptr(t, group.numel, (dt,), f"dst[{i}]") for i, t in enumerate(dsts)])
    _check(lib().tc_broadcast(group.handle, len(dsts), _dev_ptr(src, group.numel, (dt,), "src"), p, _DTYPES[dt],
                              _stream(stream)))


def broadcast_tensor(group: Group, K: int, src, dst, stream=None) -> None:
    dt = _gdt(src)
    _check(lib().tc_broadcast_tensor(group.handle, K, _dev_ptr(src, group.numel, (dt,), "src"),
                                     _dev_ptr(dst, tensor_numel(group, K), (dt,), "dst"), _DTYPES[dt],
                                     _stream(stream)))


# ----------------------------------------------------------------- pipeline

def easgd_pipeline_tensor(grads: TensorList, params: TensorList, g_tensor: Optional[torch.Tensor],
                          gbar: torch.Tensor, x: torch.Tensor, xc: torch.Tensor, eta: float, rho: float,
                          stream=None) -> None:
    """The whole step in one pass (easgd_pipeline_tensor): pack the gradient
    lists into g_tensor (skipped when None), gbar = their AVG, the fused
    elastic step on the tensor-layout workers x and the center xc, and the
    new workers unpacked into the parameter lists."""
    if grads.group is not params.group:
        raise ValueError("the gradient and parameter lists must share one group")
    group, K = grads.group, grads.K
    n = tensor_numel(group, K)
    gt = _dev_ptr(g_tensor, n, (grads.dtype,), "g_tensor") if g_tensor is not None else None
    _check(lib().easgd_pipeline_tensor(grads.handle, params.handle, gt,
                                       _dev_ptr(gbar, group.numel, (torch.float32,), "gbar"),
                                       _dev_ptr(x, n, (torch.float32,), "x"),
                                       _dev_ptr(xc, group.numel, (torch.float32,), "x_c"), float(eta), float(rho),
                                       _stream(stream)))


# --------------------------------------------------------------- layer norm

def _row_ptrs(ts, rows, cols: int, dtype: torch.dtype, device: int, what: str):
    """(device pointers, row stride in elements) of the K workers' rows."""
    if len(ts) != len(rows):
        raise ValueError(f"need {len(rows)} tensors as {what}, got {len(ts)}")
    ptrs, ld = [], None
    for k, (t, r) in enumerate(zip(ts, rows)):
        if t.get_device() != device or device < 0:
            raise _elsewhere(t, device, f"{what}[{k}]")
        if t.dtype is not dtype:
            raise TypeError(f"{what}[{k}] has dtype {t.dtype}, expected {dtype}")
        if t.shape != (r, cols):
            raise ValueError(f"{what}[{k}] has shape {tuple(t.shape)}, expected {(r, cols)}")
        if r:
            s0, s1 = t.stride()
            if s1 != 1 and cols > 1:
                raise ValueError(f"{what}[{k}]: a row's elements must be next to each other")
            if r > 1 and s0 != ld:
                if ld is not None:
                    raise ValueError(f"{what}[{k}] has a row stride of {s0}, the workers before it {ld}")
                ld = s0
        ptrs.append(t.data_ptr() if r else None)
    return _ptr_array(ptrs), cols if ld is None else ld


def _row_vectors(ts, sizes, dtypes, device: int, what: str):
    if ts is None:
        return None
    if len(ts) != len(sizes):
        raise ValueError(f"need {len(sizes)} tensors as {what}, got {len(ts)}")
    return _ptr_array([_dev_ptr(t, n, dtypes, what, device) if n else None for t, n in zip(ts, sizes)])


def _norm_rows(xs):
    if not len(xs) or any(x.dim() != 2 for x in xs):
        raise ValueError("need one [rows, columns] tensor per worker")
    if xs[0].dtype not in _DTYPES:
        raise TypeError(f"rows have dtype {xs[0].dtype}")
    rows = [x.shape[0] for x in xs]
    return (ctypes.c_int64 * len(rows))(*rows), rows, xs[0].shape[1], xs[0].dtype


def layernorm(xs: Sequence[torch.Tensor], weights, biases, ys: Sequence[torch.Tensor], means=None, rstds=None,
              eps: float = 1e-5, stream=None) -> None:
    """ys[k] = layer norm of worker k's rows xs[k] ([rows_k, columns], row
    stride free) with its own scale and shift (None: ones, zeros); means and
    rstds receive each row's statistics for the backward pass (tc_layernorm)."""
    arr, rows, cols, dt = _norm_rows(xs)
    dev = xs[0].get_device()
    xp, x_ld = _row_ptrs(xs, rows, cols, dt, dev, "x")
    yp, y_ld = _row_ptrs(ys, rows, cols, dt, dev, "y")
    wide, f32 = [cols] * len(rows), (torch.float32,)
    _check(lib().tc_layernorm(len(rows), arr, cols, xp, x_ld, _DTYPES[dt], _row_vectors(weights, wide, f32, dev, "weight"),
                              _row_vectors(biases, wide, f32, dev, "bias"), yp, y_ld, _row_vectors(means, rows, f32, dev, "mean"),
                              _row_vectors(rstds, rows, f32, dev, "rstd"), float(eps), _stream(stream)))


def layernorm_workspace(rows: Sequence[int], cols: int) -> int:
    """Bytes of workspace that layernorm_backward needs (tc_layernorm_workspace)."""
    n = lib().tc_layernorm_workspace(len(rows), (ctypes.c_int64 * max(1, len(rows)))(*[int(r) for r in rows]), int(cols))
    if n < 0:
        raise TCError(TC_EINVAL, last_error())
    return n


def _scratch(workspace: Optional[torch.Tensor], need: int, device, stream) -> torch.Tensor:
    """The caller's workspace, or one from torch's allocator that belongs to the stream the call runs on."""
    if workspace is None:
        if stream is None:
            return torch.empty(max(16, need), dtype=torch.uint8, device=device)
        s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)
        with torch.cuda.stream(s):
            return torch.empty(max(16, need), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous GPU tensor")
    return workspace


def layernorm_backward(dys: Sequence[torch.Tensor], xs: Sequence[torch.Tensor], weights, means, rstds,
                       dxs: Sequence[torch.Tensor], dweights, dbiases, workspace: Optional[torch.Tensor] = None,
                       stream=None) -> None:
    """The gradients of layernorm: dxs[k] of worker k's rows, and dweights[k],
    dbiases[k] (binary32 or bfloat16) summed over them (tc_layernorm_backward)."""
    arr, rows, cols, dt = _norm_rows(xs)
    dev = xs[0].get_device()
    dyp, dy_ld = _row_ptrs(dys, rows, cols, dt, dev, "dy")
    xp, x_ld = _row_ptrs(xs, rows, cols, dt, dev, "x")
    dxp, dx_ld = _row_ptrs(dxs, rows, cols, dt, dev, "dx")
    wide, f32 = [cols] * len(rows), (torch.float32,)
    wdt = _gdt(dweights)
    need = lib().tc_layernorm_workspace(len(rows), arr, cols)
    ws = _scratch(workspace, need, xs[0].device, stream)
    if ws.get_device() != dev:
        raise _elsewhere(ws, dev, "the workspace")
    _check(lib().tc_layernorm_backward(
        len(rows), arr, cols, dyp, dy_ld, xp, x_ld, _DTYPES[dt], _row_vectors(weights, wide, f32, dev, "weight"),
        _row_vectors(means, rows, f32, dev, "mean"), _row_vectors(rstds, rows, f32, dev, "rstd"), dxp, dx_ld,
        _row_vectors(dweights, wide, (wdt,), dev, "dweight"), _row_vectors(dbiases, wide, (wdt,), dev, "dbias"), _DTYPES[wdt],
        ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))


# ------------------------------------------------------- orthogonalised update

class OrthoPlan:
    """Which tensors of a group are matrices: shapes[t] is (rows, columns), or
    None for a tensor whose update is taken as it is; scales[t] multiplies
    tensor t's update (None: ones).  For K copies (tc_ortho_create)."""

    def __init__(self, group: Group, K: int, shapes, scales: Optional[Sequence[float]] = None):
        if len(shapes) != group.n:
            raise ValueError(f"need {group.n} shapes, got {len(shapes)}")
        if scales is not None and len(scales) != group.n:
            raise ValueError(f"need {group.n} scales, got {len(scales)}")
        sides = [(0, 0) if s is None else (int(s[0]), int(s[1])) for s in shapes]
        rows, cols = [(ctypes.c_int64 * group.n)(*[s[i] for s in sides]) for i in range(2)]
        factors = None if scales is None else (ctypes.c_float * group.n)(*[float(s) for s in scales])
        h = lib().tc_ortho_create(group.handle, int(K), rows, cols, factors)
        if not h:
            raise TCError(TC_EINVAL, last_error())
        self._h = h
        self.group, self.K = group, int(K)
        self.workspace = lib().tc_ortho_workspace(h)

    @property
    def handle(self):
        return self._h

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.tc_ortho_destroy(h)


def ortho_workspace(plan: OrthoPlan) -> int:
    """Bytes of workspace that orthogonalize needs (tc_ortho_workspace)."""
    return plan.workspace


def orthogonalize(plan: OrthoPlan, gs: Sequence[torch.Tensor], outs: Sequence[torch.Tensor],
                  momenta: Optional[Sequence[torch.Tensor]] = None, mu: float = 0.95, nesterov: bool = True,
                  steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """outs[k] = the momentum update of the flat gradient gs[k], its matrices
    orthogonalised by Newton-Schulz steps; momenta (binary32) are updated in
    place (None: the gradient itself is the update).  coefficients: (a, b, c)
    for every step, or one triple a step (tc_orthogonalize)."""
    n = plan.group.numel
    if len(gs) != plan.K or len(outs) != plan.K or (momenta is not None and len(momenta) != plan.K):
        raise ValueError(f"need {plan.K} gradients, updates and momenta")
    triples = coefficients if hasattr(coefficients[0], "__len__") else [coefficients] * int(steps)
    if len(triples) != int(steps) or any(len(t) != 3 for t in triples):
        raise ValueError(f"need three coefficients, or three for each of the {steps} steps")
    coeff = (ctypes.c_float * (3 * len(triples)))(*[float(v) for t in triples for v in t])
    gdt, odt = _gdt(gs), _gdt(outs)
    gp = _ptr_array([_dev_ptr(t, n, (gdt,), f"grad[{k}]") for k, t in enumerate(gs)])
    op = _ptr_array([_dev_ptr(t, n, (odt,), f"out[{k}]") for k, t in enumerate(outs)])
    mp = None if momenta is None else _ptr_array([_dev_ptr(t, n, (torch.float32,), f"momentum[{k}]") for k, t in enumerate(momenta)])
    ws = _scratch(workspace, plan.workspace, gs[0].device, stream)
    _check(lib().tc_orthogonalize(plan.handle, gp, _DTYPES[gdt], mp, float(mu), int(bool(nesterov)), op, _DTYPES[odt],
                                  int(steps), coeff, float(eps), ws.data_ptr(), ws.numel() * ws.element_size(),
                                  _stream(stream)))
