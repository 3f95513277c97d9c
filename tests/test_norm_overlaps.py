"""Which buffers the layer norm's calls may share, by addresses alone: a call
that is refused never reaches a device.  Only where there is no GPU, because
the addresses are made up: there a call that is not refused ends with the
device's error."""

import ctypes

import pytest
import torch

import paper_1801_03855_amd as tc

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses")

COLS, LD, ROWS = 64, 96, (8, 1, 5)
BUFFERS = ("x", "y", "weight", "bias", "mean", "rstd", "dy", "dx", "dweight", "dbias")
WRITTEN = {"forward": ("y", "mean", "rstd"), "backward": ("dx", "dweight", "dbias", "workspace")}
READ = {"forward": ("x", "weight", "bias"), "backward": ("x", "dy", "weight", "mean", "rstd")}


def size(name, k):
    if name in ("x", "y", "dy", "dx"):
        return ((ROWS[k] - 1) * LD + COLS) * 4
    return ROWS[k] * 4 if name in ("mean", "rstd") else COLS * 4


def apart():
    """Every buffer of every worker, a page from the next, and the workspace."""
    at = {(n, k): 0x10000 * (1 + BUFFERS.index(n) * 4 + k) for n in BUFFERS for k in range(3)}
    at["workspace", 0] = 0x4000000
    return at


def call(which, at, rows=ROWS, ld=LD):
    L = tc.lib()
    counts = (ctypes.c_int64 * 3)(*rows)
    p = {n: (ctypes.c_void_p * 3)(*[at[n, k] for k in range(3)]) for n in BUFFERS}
    if which == "forward":
        status = L.tc_layernorm(3, counts, COLS, p["x"], ld, 0, p["weight"], p["bias"], p["y"], ld, p["mean"], p["rstd"], 1e-5, None)
    else:
        status = L.tc_layernorm_backward(3, counts, COLS, p["dy"], ld, p["x"], ld, 0, p["weight"], p["mean"], p["rstd"], p["dx"], ld,
                                         p["dweight"], p["dbias"], 0, at["workspace", 0], 1 << 20, None)
    return status, tc.last_error()


def refused(which, at, **kw):
    status, text = call(which, at, **kw)
    return status == tc.TC_EINVAL and "overlaps" in text


def everything(which):
    return [(n, k) for n in WRITTEN[which] + READ[which] for k in range(1 if n == "workspace" else 3)]


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_buffers_apart_are_not_refused(which):
    assert call(which, apart())[0] not in (0, tc.TC_EINVAL)


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_nothing_written_shares_its_first_or_last_bytes(which):
    for w in everything(which):
        if w[0] not in WRITTEN[which]:
            continue
        need = tc.lib().tc_layernorm_workspace(3, (ctypes.c_int64 * 3)(*ROWS), COLS) if w[0] == "workspace" else size(*w)
        for other in everything(which):
            if other == w:
                continue
            for place in ("first", "last"):
                if other[0] == "workspace" and place == "last":
                    continue
                at = apart()
                step = 256 if w[0] == "workspace" else 4
                # the last bytes of `other` are the first ones of `w`
                at[w] = at[other] if place == "first" else (at[other] + size(*other) - 1) // step * step
                if at[w] + need <= at[other]:
                    continue
                rows_in_place = {w[0], other[0]} in ({"x", "y"}, {"x", "dx"}, {"dy", "dx"}) and w[1] == other[1] and place == "first"
                assert refused(which, at) != rows_in_place, (which, w, other, place, call(which, at))


@pytest.mark.parametrize("which,rows,name", [("forward", "x", "mean"), ("forward", "y", "bias"), ("backward", "dy", "dweight"),
                                             ("backward", "x", "workspace"), ("backward", "dx", "rstd")])
def test_a_block_between_rows_shares_nothing(which, rows, name):
    """Worker 0's eight rows have 32 elements between them."""
    wide = 4096  # so that every buffer here fits between two rows
    at = apart()
    for n in ("x", "y", "dy", "dx"):
        for k in range(3):
            at[n, k] = 0x10000000 * (1 + BUFFERS.index(n) * 4 + k)
    base = at[rows, 0]
    n = size(name, 0) if name != "workspace" else tc.lib().tc_layernorm_workspace(3, (ctypes.c_int64 * 3)(*ROWS), COLS)
    step = 256 if name == "workspace" else 4
    assert n + 1024 < (wide - COLS) * 4
    for row in (0, 3, 6):
        begin, end = base + (row * wide + COLS) * 4, base + (row + 1) * wide * 4
        for place, bad in ((begin, False), ((end - n) // step * step, False), (begin - step, True), ((end - n) // step * step + step, True)):
            at[name, 0] = place
            assert refused(which, at, ld=wide) == bad, (row, hex(place - base))
    at[name, 0] = base + (7 * wide + COLS) * 4  # behind the last row
    assert not refused(which, at, ld=wide)


def test_a_worker_without_rows_needs_no_place():
    at = apart()
    at["mean", 1] = at["y", 0]
    assert refused("forward", at) and not refused("forward", at, rows=(8, 0, 5))
    at = apart()
    at["dx", 2] = at["weight", 0]
    assert refused("backward", at) and not refused("backward", at, rows=(8, 1, 0))
    at["dweight", 2] = at["weight", 0]  # which it still writes
    assert refused("backward", at, rows=(8, 1, 0))
