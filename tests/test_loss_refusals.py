"""What the cross entropy's and the dropout's calls refuse, by arguments and
addresses alone: a call that is refused never reaches a device.  Only where there
is no GPU, because the addresses are made up: there a call that is not refused
ends with the device's error."""

import ctypes

import pytest
import torch

import paper_1801_03855_amd as tc
from tests.test_norm_device import Rows

without_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up addresses")

COLS, CLASSES, LD, ROWS = 64, 100, 96, (8, 0, 5)
NAMES = ("x", "weight", "bias", "label", "loss", "lse", "dloss", "dx", "dweight", "dbias", "residual", "y")
READ = {"ce": ("x", "weight", "bias", "label"), "grad": ("x", "weight", "bias", "label", "lse", "dloss"), "dropout": ("x", "residual"),
        "dropout_grad": ("x",)}
WRITTEN = {"ce": ("loss", "lse"), "grad": ("dx", "dweight", "dbias"), "dropout": ("y",), "dropout_grad": ("y",)}
NEED = 1 << 24


def places():
    at = {(n, k): 0x40000000 + 0x100000 * (NAMES.index(n) * 4 + k) for n in NAMES for k in range(3)}
    return at | {("workspace", 0): 0x20000000, ("random", 0): 0x10000000}


def call(which, at=None, K=3, rows=ROWS, cols=COLS, classes=CLASSES, ld=LD, dtype=0, w_dtype=0, dw_dtype=0, p=0.1, site=0, scale=1.0,
         space=NEED, null=()):
    at = at or places()
    L = tc.lib()
    counts = (ctypes.c_int64 * 3)(*rows)
    v = {n: None if n in null else (ctypes.c_void_p * 3)(*[at[n, k] for k in range(3)]) for n in NAMES}
    ws, random = [None if n in null else at[n, 0] for n in ("workspace", "random")]
    if which == "ce":
        status = L.tc_cross_entropy(K, counts, cols, classes, v["x"], ld, dtype, v["weight"], v["bias"], w_dtype, v["label"], v["loss"], v["lse"],
                                    ws, space, None)
    elif which == "grad":
        status = L.tc_cross_entropy_backward(K, counts, cols, classes, v["x"], ld, dtype, v["weight"], v["bias"], w_dtype, v["label"], v["lse"],
                                             v["dloss"], scale, v["dx"], ld, v["dweight"], v["dbias"], dw_dtype, ws, space, None)
    elif which == "dropout":
        status = L.tc_dropout(K, counts, cols, v["x"], ld, dtype, v["residual"], ld, v["y"], ld, p, random, site, None)
    else:
        status = L.tc_dropout_backward(K, counts, cols, v["x"], ld, dtype, v["y"], ld, p, random, site, None)
    return status, tc.last_error()


CALLS = ("ce", "grad", "dropout", "dropout_grad")


@without_gpu
@pytest.mark.parametrize("which", CALLS)
def test_a_good_call_reaches_the_device(which):
    assert call(which)[0] == tc.TC_EHIP
    optional = {"ce": ("bias",), "grad": ("bias", "dloss", "dbias"), "dropout": ("residual",), "dropout_grad": ()}[which]
    for name in optional:
        assert call(which, null=(name,))[0] == tc.TC_EHIP
    # a worker without rows needs no pointers, except for the gradients of its parameters
    at = places()
    for n in NAMES:
        if n not in ("dweight", "dbias"):
            at[n, 1] = None
    assert call(which, at)[0] == tc.TC_EHIP


@without_gpu
@pytest.mark.parametrize("which", CALLS)
def test_arguments(which):
    bad = [dict(K=0), dict(K=65), dict(cols=0), dict(rows=(8, -1, 5)), dict(ld=COLS - 1), dict(dtype=2), dict(null=("x",))]
    if which in ("ce", "grad"):
        bad += [dict(classes=0), dict(classes=(1 << 24) + 1), dict(cols=(1 << 18) + 1, ld=1 << 19), dict(w_dtype=7), dict(rows=((1 << 24) + 1, 0, 1)),
                dict(rows=(1 << 24, 0, 1), cols=1 << 13, ld=1 << 13), dict(classes=1 << 24, cols=1 << 13, ld=1 << 13),
                dict(space=255), dict(null=("workspace",)), dict(null=("weight",)), dict(null=("label",)), dict(null=("lse",))]
    if which == "ce":
        bad += [dict(null=("loss",))]
    if which == "grad":
        bad += [dict(dw_dtype=-1), dict(scale=float("inf")), dict(scale=float("nan")), dict(null=("dx",)), dict(null=("dweight",))]
    if which.startswith("dropout"):
        bad += [dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(site=-1), dict(site=65536), dict(null=("random",)), dict(null=("y",)),
                dict(rows=(1 << 43, 0, 1))]
    for kw in bad:
        status, text = call(which, **kw)
        assert status == tc.TC_EINVAL and text, kw


@without_gpu
@pytest.mark.parametrize("which", CALLS)
def test_null_and_misaligned_pointers(which):
    names = READ[which] + WRITTEN[which]
    for name in names:
        at = places()
        at[name, 2] = None
        assert call(which, at)[0] == tc.TC_EINVAL, name
        at = places()
        at[name, 2] += 1
        status, text = call(which, at)
        assert status == tc.TC_EINVAL and "aligned" in text, name
    at = places()
    if which in ("ce", "grad"):
        at["workspace", 0] += 128
    else:
        at["random", 0] += 4
    assert call(which, at)[0] == tc.TC_EINVAL


def size(name, k, which):
    if name in ("x", "dx", "residual", "y"):
        return ((ROWS[k] - 1) * LD + COLS) * 4
    if name == "workspace":
        return (tc.cross_entropy_workspace if which == "ce" else tc.cross_entropy_backward_workspace)(ROWS, COLS, CLASSES)
    if name == "random":
        return 16
    return {"weight": CLASSES * COLS * 4, "dweight": CLASSES * COLS * 4, "bias": CLASSES * 4, "dbias": CLASSES * 4, "label": ROWS[k] * 8}.get(name, ROWS[k] * 4)


@without_gpu
@pytest.mark.parametrize("which", CALLS)
def test_what_is_written_shares_nothing(which):
    extra = "workspace" if which in ("ce", "grad") else "random"
    places_of = [(n, k) for n in READ[which] + WRITTEN[which] for k in (0, 2)] + [(extra, 0)]
    written = [p for p in places_of if p[0] in WRITTEN[which] or p[0] == "workspace"]
    for w in written:
        for other in places_of:
            if other == w:
                continue
            own_rows = {("x", "dx"), ("x", "y"), ("residual", "y")}
            rows = w[0] in ("dx", "y") and (other[0], w[0]) in own_rows
            at = places()
            if other[0] == "workspace" or w[0] == "random":
                continue
            at[other] = at[w]
            status, text = call(which, at)
            if rows and other[1] == w[1]:
                assert status == tc.TC_EHIP, (w, other)  # in place
            else:
                assert status == tc.TC_EINVAL and "overlaps" in text, (w, other)
            # the last element of one in the first of the other
            at = places()
            unit = 8 if other[0] in ("label", "random") else 4
            at[other] = at[w] + (size(*w, which) - unit) // unit * unit
            status, text = call(which, at)
            assert status == tc.TC_EINVAL and "overlaps" in text, (w, other)


@without_gpu
def test_what_is_read_may_be_shared():
    for which in ("ce", "grad"):
        at = places()
        for n in READ[which]:
            at[n, 2] = at[n, 0]
        assert call(which, at)[0] == tc.TC_EHIP


def test_workspaces():
    for bad in (dict(rows=[-1]), dict(cols=0), dict(classes=0)):
        a = {"rows": [4], "cols": 8, "classes": 16} | bad
        with pytest.raises(tc.TCError):
            tc.cross_entropy_workspace(**a)
        with pytest.raises(tc.TCError):
            tc.cross_entropy_backward_workspace(**a)
    small = tc.cross_entropy_workspace([4, 0], 64, 1000)
    assert 0 < small < tc.cross_entropy_backward_workspace([4, 0], 64, 1000)
    # less than half of what the logits of a large batch would take in 16 bits, and than g both ways
    rows, classes = 8192, 131072
    assert tc.cross_entropy_workspace([rows], 4096, classes, torch.bfloat16, torch.bfloat16) < rows * classes
    assert tc.cross_entropy_backward_workspace([rows], 4096, classes, torch.bfloat16, torch.bfloat16, torch.bfloat16) < 4 * rows * classes


class Tensors(Rows):
    def __init__(self, device, *shape, dtype=torch.float32):
        super().__init__(device, *shape)
        self.dtype = dtype

    @property
    def nbytes(self):
        return self.numel() * 4


@pytest.fixture
def recorded(monkeypatch):
    """The calls that reach the library."""
    calls = []

    class Library:
        def __getattr__(self, name):
            def f(*a):
                if name.endswith("workspace"):
                    return 4096
                calls.append(name)
                return 0
            return f

    monkeypatch.setattr(tc, "lib", lambda: Library())
    monkeypatch.setattr(tc, "_stream", lambda stream: 0)
    return calls


def python_call(which, **change):
    i64 = torch.int64
    t = {"x": (4, 64), "w": (10, 64), "b": (10,), "label": (4,), "loss": (4,), "lse": (4,), "dloss": (4,), "dx": (4, 64), "dw": (10, 64),
         "db": (10,), "r": (4, 64), "y": (4, 64)}
    v = {n: [Tensors(0, *s, dtype=i64 if n == "label" else torch.float32) for _ in range(2)] for n, s in t.items()}
    v["workspace"], v["random"] = Tensors(0, 4096), Tensors(0, 2, dtype=i64)
    for n, new in change.items():
        v[n] = new if n in ("workspace", "random") else [v[n][0], new]
    if which == "ce":
        tc.cross_entropy(v["x"], v["w"], v["b"], v["label"], v["loss"], v["lse"], workspace=v["workspace"])
    elif which == "grad":
        tc.cross_entropy_backward(v["x"], v["w"], v["b"], v["label"], v["lse"], v["dloss"], v["dx"], v["dw"], v["db"], workspace=v["workspace"])
    elif which == "dropout":
        tc.dropout(v["x"], v["r"], v["y"], v["random"])
    else:
        tc.dropout_backward(v["x"], v["y"], v["random"])


PYTHON = [("ce", n) for n in ("x", "w", "b", "label", "loss", "lse", "workspace")]
PYTHON += [("grad", n) for n in ("x", "w", "b", "label", "lse", "dloss", "dx", "dw", "db", "workspace")]
PYTHON += [("dropout", n) for n in ("x", "r", "y", "random")] + [("dropout_grad", n) for n in ("x", "y", "random")]


@without_gpu
@pytest.mark.parametrize("which,name", PYTHON)
def test_one_tensor_elsewhere_or_of_another_kind(recorded, which, name):
    python_call(which)
    assert len(recorded) == 1
    shape = {"x": (4, 64), "r": (4, 64), "y": (4, 64), "dx": (4, 64), "w": (10, 64), "dw": (10, 64), "b": (10,), "db": (10,),
             "workspace": (4096,), "random": (2,)}.get(name, (4,))
    own = torch.int64 if name in ("label", "random") else torch.float32
    with pytest.raises(ValueError):
        python_call(which, **{name: Tensors(1, *shape, dtype=own)})
    if name != "workspace":
        with pytest.raises((TypeError, ValueError)):
            python_call(which, **{name: Tensors(0, *shape, dtype=torch.float16)})
        if name != "x":
            with pytest.raises(ValueError):
                python_call(which, **{name: Tensors(0, *[s + 1 for s in shape], dtype=own)})
    assert len(recorded) == 1
