"""The hand-overs of the loss and of the weights' update through LDS, as test_lds_exchange reads them: every access that another lane of the wavefront follows up is behind a fence."""
import os
import re
import subprocess

import pytest

from paper_2605_29346_amd import build

CSRC = os.path.join(build.HERE, "csrc")


@pytest.mark.parametrize("source,function,fences", [("zg_loss.hip", "hand_over_dz", 2), ("zg_orthogonal.hip", "hand_over_step", 4)])
def test_cells_that_lanes_exchange_are_fenced(tmp_path, source, function, fences):
    cc = build.hipcc()
    if cc is None:
        pytest.skip("no hipcc here")
    out = tmp_path / "code.ll"
    subprocess.run([cc, "-x", "hip", "--offload-arch=gfx950", "--cuda-device-only", "-O3", "-std=c++17", "-I", os.path.join(build.ROOT, "include"), "-I", CSRC, "-S", "-emit-llvm", "-Xclang",
                    "-disable-llvm-passes", os.path.join(CSRC, source), "-o", str(out)], check=True, capture_output=True)
    functions = dict(re.findall(r"^define [^\n]*?@(\S+?)\([^\n]*\n(.*?)^}", out.read_text(), re.M | re.S))
    bodies = [body for name, body in functions.items() if function in name and "lds_exchange" in body]
    assert len(bodies) >= 4
    for body in bodies:
        at = [m.start() for m in re.finditer(r"call void @\S*lds_exchange", body)]
        places = set(re.findall(r"(%\S+) = getelementptr", body))  # (what is stored to elsewhere are variables of the function's own)
        writes = [m.start() for m in re.finditer(r"store <4 x float> %\S+, ptr (%\S+),", body) if m.group(1) in places]
        reads = [m.start() for m in re.finditer(r"load <4 x float>, ptr (%\S+),", body) if m.group(1) in places]
        assert len(at) == fences
        # cells go in before the first fence and are read between the first and the second; where they are turned, they go in once more before the third, and are read between that and the fourth
        assert min(writes) < at[0] < min(reads) and max(reads) < at[1] and not any(at[0] < w < at[1] for w in writes)
        if fences == 4:
            assert any(at[1] < w < at[2] for w in writes) and max(writes) < at[2]
            assert any(at[2] < m.start() < at[3] for m in re.finditer(r"load float, ptr %", body)) and not re.search(r"load float, ptr %", body[at[3]:])
