"""The waits of the orthogonalised update's products, in the machine code that
this project's compiler makes of them (no GPU).

A kernel with more than two stages has loads into LDS under way when its main
loop ends.  Its result is then written over the same LDS, so between the last
such load and the first such write every wave has to wait for its loads, by a
wait that the source itself states, and meet the others at a barrier."""

import os
import re
import shutil
import subprocess

import pytest

from paper_1801_03855_amd import build as b


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: lines} of the product kernels."""
    if not (os.path.exists(b.HIPCC) or shutil.which(b.HIPCC)):
        pytest.skip("no hipcc here")
    out = str(tmp_path_factory.mktemp("asm") / "tc_ortho.s")
    flags = [f for f in b.FLAGS if f not in ("-shared", "-Wall")]
    subprocess.run([b.HIPCC, *flags, "-I", b.INCLUDE, "-I", b.CSRC, "--offload-device-only", "-S",
                    os.path.join(b.CSRC, "tc_ortho.hip"), "-o", out], check=True, stderr=subprocess.DEVNULL)
    found, name = {}, None
    for line in open(out):
        if m := re.match(r"(_Z\w*ortho_gemm_kernel\w*):", line):
            name = m.group(1)
            found[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name:
            found[name].append(line.strip())
    assert found
    return found


def test_no_load_is_under_way_where_the_tile_is_written(kernels):
    checked = 0
    for name, lines in kernels.items():
        last_load = max(i for i, s in enumerate(lines) if s.startswith("global_load_lds"))
        first_write = next(i for i in range(last_load, len(lines)) if lines[i].startswith("ds_write"))
        between = lines[last_load:first_write]
        # loads of more than one stage stay under way over a barrier in the loop
        if not any(s.startswith("s_waitcnt vmcnt(") and "vmcnt(0)" not in s for s in lines[:first_write] if "lgkmcnt(0)" in s):
            continue
        checked += 1
        stated = [i for i, s in enumerate(between) if s.startswith(";;#ASMSTART")
                  and re.fullmatch(r"s_waitcnt vmcnt\(0\)( lgkmcnt\(0\))?", between[i + 1])]
        assert stated, f"{name}: no wait for the loads under way is stated"
        assert any(s == "s_barrier" for s in between[stated[-1]:]), f"{name}: no barrier after the wait"
    assert checked
