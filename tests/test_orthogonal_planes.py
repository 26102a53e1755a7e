"""Which results are made of fp16 operands, asked of the library's own launches (without a device), and what those operands leave, by the operator's documented arithmetic in 64 bits: no more than is stated."""
import json
import os
import re
import subprocess
import sys

import pytest
import torch

import orthogonal_util as O
from test_gpu_orthogonal_coefficients import FAST, SAFE, SETS, STATED

_ASK = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)
shim.launched_kernels.restype = C.c_char_p
sys.path.insert(0, "tests")
from paper_2605_29346_amd import zg
L, n, out = zg.lib(), C.c_size_t(), []
for rows, cols, kind, k in json.loads(sys.argv[2]):
    flat = (C.c_float * (3 * len(k)))(*(v for t in k for v in t))
    a = zg.OrthogonalizeArgs(rows=rows, cols=cols, dtype=zg.F32, out_dtype=kind, steps=len(k), eps=1e-7, coefficients=C.addressof(flat), d_G=1 << 44, ld_G=cols, d_O=2 << 44, ld_O=cols)
    assert L.zg_orthogonalize_workspace(C.byref(a), C.byref(n)) == 0, L.zg_last_error()
    assert L.zg_orthogonalize(C.byref(a), 3 << 44, n.value, None) == 0, L.zg_last_error()
    out.append([n.value, shim.launched_kernels().decode().split()])
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    shim = tmp_path_factory.mktemp("shim") / "kernel_shim.so"
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(root, "tests", "kernel_shim.cpp"), "-o", str(shim), "-ldl"], check=True)

    def asked(cases):
        """(workspace bytes, whether single planes are the operands) of each (rows, cols, type, triples)"""
        run = subprocess.run([sys.executable, "-c", _ASK, str(shim), json.dumps(cases)], cwd=root, timeout=100, capture_output=True, text=True)
        assert run.returncode == 0, run.stderr[-2000:]
        got = []
        for size, launched in json.loads(run.stdout):
            planes = {m.group(1) for m in (re.search(r"\d+k_step_[a-z0-9]+?ILi([13])E", name) for name in launched) if m}
            assert len(planes) == 1, launched
            got.append((size, planes == {"1"}))
        return got
    return asked


BF16 = 4
MANY = dict(SETS)
MANY.update({f"default {n}": [O.MUON] * n for n in (1, 2, 3, 7)} | {f"fast {n}": FAST[:n] for n in (1, 2, 3, 4)} | {f"safe {n}": SAFE[:n] for n in (1, 2, 4)})
MANY.update({"shrinking": [(0.5, 0.0, 0.0)] * 2, "cubes": [(0.0, 1.0, 0.0)] * 3, "turned over": [(-1.5, 0.5, 0.0)] * 4, "steep at the top": [(3.0, -4.0, 1.5)] * 6, "linear": [(2.0, 0.0, 0.0)] * 6, "ends at 0": [(1.0, -1.0, 0.0)] * 2})


@pytest.fixture(scope="module")
def single(ask):
    return dict(zip(MANY, (one for _, one in ask([(256, 256, BF16, k) for k in MANY.values()]))))


def test_the_usual_steps_take_single_planes_and_steep_ones_do_not(single):
    for name in ("default", "default 4", "default 1", "cubic 6", "quintic 6", "turned over", "linear"):
        assert single[name], name
    for name in ("default 6", "default 7", "fast", "fast 3", "safe", "safe 3", "safe 4", "shrinking", "cubes", "steep at the top"):
        assert not single[name], name


def _matrices(rows, cols):
    g = torch.Generator().manual_seed(rows + cols)
    noise = torch.randn(rows, cols, generator=g)
    yield "noise", noise
    yield "one direction", torch.randn(rows, 1, generator=g) @ torch.randn(1, cols, generator=g) + 0.05 * noise
    u, v = torch.linalg.qr(torch.randn(rows, rows, generator=g))[0], torch.linalg.qr(torch.randn(cols, rows, generator=g))[0]
    yield "falling", u @ torch.diag(1.0 / torch.arange(1, rows + 1)) @ v.t()
    yield "even", u @ v.t()


@pytest.mark.parametrize("name", MANY)
def test_single_planes_leave_what_is_stated(single, name, monkeypatch):
    if not single[name]:
        return
    monkeypatch.setattr(O, "single", lambda *_: True)
    k = MANY[name]
    for size in ((256, 256), (256, 900), (400, 400)):
        for what, m in _matrices(*size):
            want = O.exact(m, len(k), k)
            off = float((O.emulated(m, torch.bfloat16, len(k), k) - want).norm()) / size[0] ** 0.5
            assert off <= STATED, (size, what, off)


def test_a_workspace_goes_by_the_matrix_and_not_by_the_steps(ask):
    for rows, cols in ((256, 256), (300, 2000), (1024, 4096), (2300, 700)):
        sizes = {size for size, _ in ask([(rows, cols, BF16, k) for k in MANY.values()])}
        assert len(sizes) == 1, (rows, cols, sizes)
