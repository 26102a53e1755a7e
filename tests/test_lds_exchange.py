"""Lanes of a wavefront hand cells to each other through LDS without a workgroup barrier: what holds the compiler to the order of those accesses
is read from the code as the front end leaves it, before anything is moved."""
import os
import re
import subprocess

import pytest

from paper_2605_29346_amd import build

SOURCE = os.path.join(build.HERE, "csrc", "zg_linear.hip")


def _functions(tmp_path):
    cc = build.hipcc()
    if cc is None:
        pytest.skip("no hipcc here")
    out = tmp_path / "linear.ll"
    subprocess.run([cc, "-x", "hip", "--offload-arch=gfx950", "--cuda-device-only", "-O3", "-std=c++17", "-I", os.path.join(build.ROOT, "include"), "-I",
                    os.path.dirname(SOURCE), "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes", SOURCE, "-o", str(out)], check=True, capture_output=True)
    return dict(re.findall(r"^define [^\n]*?@(\S+?)\([^\n]*\n(.*?)^}", out.read_text(), re.M | re.S))


def test_cells_that_lanes_exchange_are_fenced(tmp_path):
    functions = _functions(tmp_path)
    fence = [body for name, body in functions.items() if "lds_exchange" in name]
    assert len(fence) == 1
    order = [re.search(p, fence[0]) for p in (r'fence syncscope\("wavefront"\) release', r"call void @llvm\.amdgcn\.wave\.barrier", r'fence syncscope\("wavefront"\) acquire')]
    assert all(order) and [m.start() for m in order] == sorted(m.start() for m in order)
    bodies = [body for name, body in functions.items() if "hand_over" in name and re.search(r"call void @\S*N_16finish", body)]  # (functions, or lambdas in them)
    assert len(bodies) >= 10
    for body in bodies:
        writes = [m.start() for m in re.finditer(r"store <4 x float>", body)]
        fences = [m.start() for m in re.finditer(r"call void @\S*lds_exchange", body)]
        reads = [m.start() for m in re.finditer(r"call void @\S*N_16finish", body)]  # (its argument reads the cells)
        assert len(reads) == 1 and len(fences) == 2 and writes
        assert max(writes) < fences[0] < reads[0] < fences[1]
