"""Tiles that a wave turns in LDS: what its lanes write and others of them read is ordered for the compiler too, which need not keep a store in front of another lane's load
(the two are at different addresses of a lane)."""
import os
import re
import subprocess

import pytest

from paper_2603_11564_amd import build

WIDE = re.compile(r"(store|= load) <4 x i32>.*ptr addrspace\(3\)")
ORDERS = re.compile(r"^\s*fence |@llvm\.amdgcn\.s\.barrier|@llvm\.amdgcn\.wave\.barrier")


def unordered(lines):
    """Pairs of a 16-byte LDS store and a load, or a load and a store behind it, with nothing between them that orders memory, in a basic block."""
    found, last = [], None
    for line in lines:
        if re.match(r"^[\w.$-]+:", line) or ORDERS.search(line):
            last = None
            continue
        m = WIDE.search(line)
        if m:
            kind = m.group(1)
            if last is not None and last != kind:
                found.append(line.strip())
            last = kind
    return found


def test_the_scan_itself():
    store, load = "  store <4 x i32> %a, ptr addrspace(3) %p, align 16", "  %x = load <4 x i32>, ptr addrspace(3) %q, align 16"
    fence = '  fence syncscope("wavefront") acq_rel'
    assert unordered([store, store, load, load]) == [load.strip()] and unordered([load, store]) == [store.strip()]
    assert unordered([store, fence, load, fence, store]) == [] and unordered([store, "5:                                  ; preds = %4", load]) == []
    assert unordered([store, "  tail call void @llvm.amdgcn.s.barrier()", load]) == []


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Intermediate code of the kernels of paged_blocks.hip, lines by name."""
    out = str(tmp_path_factory.mktemp("ir") / "paged_blocks.ll")
    r = subprocess.run([build._hipcc(), *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, "paged_blocks.hip"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    found, name = {}, None
    for line in open(out):
        m = re.match(r"define .*@(\w+)\(", line)
        if m:
            name = m.group(1)
            found[name] = []
        elif name is not None:
            found[name].append(line.rstrip())
    return found


def test_turned_tiles_are_fenced(kernels):
    scores = {name: lines for name, lines in kernels.items() if "paged_scores_kernel" in name}
    assert len(scores) == 6
    for name, lines in scores.items():
        kinds = [m.group(1) for line in lines if (m := WIDE.search(line))]
        assert kinds.count("store") >= 4 and kinds.count("= load") >= 4, name
        assert not unordered(lines), (name, unordered(lines)[:2])
        assert sum("fence" in line and 'syncscope("wavefront")' in line for line in lines) >= 2, name
