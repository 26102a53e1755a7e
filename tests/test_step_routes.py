"""The sizes of the GPU tests reach every kernel of the loss and of the weights' update: asked of the library's own launches, with the runtime's launch call replaced by one that writes their names down.  No
device is needed and nothing is run."""
import json
import os
import re
import subprocess
import sys

import pytest

_ASK = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)
shim.launched_kernels.restype = shim.registered_kernels.restype = C.c_char_p
sys.path.insert(0, "tests")
from paper_2605_29346_amd import zg
import test_gpu_loss as T
import test_gpu_orthogonal as O
L = zg.lib()
SIZE = {zg.F32: 4, zg.F16: 2, zg.BF16: 2}
at = lambda i: i << 44  # (addresses that nobody looks at, far from each other)
out = {"registered": shim.registered_kernels().decode().split("\n"), "launched": []}
def note(status, *what):
    assert status == 0, (status, L.zg_last_error(), what)
    out["launched"].append([list(what), shim.launched_kernels().decode().split()])
for t in SIZE:
    for rows, k, n, pad, shift in T.SIZES + T.ROUTES:
        ld, off, weight = k + pad, shift * SIZE[t], at(5) if pad else None
        a = zg.LossArgs(rows=rows, in_=k, out=n, dtype=t, label_dtype=zg.I64, d_A=at(1) + off, ld_A=ld, d_W=at(2) + off, ld_W=ld, d_labels=at(3), d_weight=weight, d_loss=at(6), d_lse=at(7))
        note(L.zg_linear_cross_entropy(C.byref(a), at(8), 1 << 43, None), "loss", t, rows, k, n, pad)
        b = zg.LossGradArgs(rows=rows, in_=k, out=n, dtype=t, label_dtype=zg.I64, d_A=at(1) + off, ld_A=ld, d_W=at(2) + off, ld_W=ld, d_labels=at(3), d_weight=weight, d_lse=at(7), d_dA=at(9), ld_dA=k,
                            d_dW=at(10), ld_dW=k, d_dbias=at(11))
        note(L.zg_linear_cross_entropy_backward(C.byref(b), at(8), 1 << 43, None), "gradients", t, rows, k, n, pad)
K = (C.c_float * 15)(*([3.4445, -4.7750, 2.0315] * 5))
for t in SIZE:
    for o in SIZE:
        for rows, cols, pad, shift in O.SIZES + O.ROUTES:
            a = zg.OrthogonalizeArgs(rows=rows, cols=cols, dtype=t, out_dtype=o, steps=5, eps=1e-7, coefficients=C.addressof(K), d_G=at(1), ld_G=cols, d_O=at(2), ld_O=cols)
            note(L.zg_orthogonalize(C.byref(a), at(8), 1 << 43, None), "orthogonalize", o, rows, cols)
b = zg.LossGradArgs(rows=0, in_=8, out=8, dtype=zg.F32, label_dtype=zg.I64, d_dW=at(10), ld_dW=8)
note(L.zg_linear_cross_entropy_backward(C.byref(b), at(8), 1 << 43, None), "no rows")
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def asked(tmp_path_factory):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    shim = tmp_path_factory.mktemp("shim") / "kernel_shim.so"
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(root, "tests", "kernel_shim.cpp"), "-o", str(shim), "-ldl"], check=True)
    run = subprocess.run([sys.executable, "-c", _ASK, str(shim)], cwd=root, timeout=100, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-2000:]
    return json.loads(run.stdout)


def test_every_kernel_is_reached(asked):
    every = {n for n in asked["registered"] if re.search(r"\d+k_(loss|step|start)_", n)}
    reached = {n for _, launched in asked["launched"] for n in launched}
    assert len(every) > 70
    assert sorted(every - reached) == []


def test_the_loss_takes_two_launches_or_three_and_an_update_one_or_three_a_step(asked):
    for what, launched in asked["launched"]:
        own = [n for n in launched if re.search(r"\d+k_(loss|step|start)_", n) and "k_loss_pack" not in n]
        if what[0] == "loss":
            assert len(own) in (2, 3), (what, own)
        elif what[0] == "orthogonalize":
            small = min(what[2:]) <= 64 and max(what[2:]) <= 384
            assert len(own) == len(launched) == (1 if small else 17), (what, own)
