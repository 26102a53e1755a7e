"""The sizes of test_gpu_loss_row_pieces are made of the pieces that they are meant for, others are not.  Asked of the library's own launches, without a device."""
import json
import os
import subprocess
import sys

import pytest
import torch

from test_gpu_loss_row_pieces import SIZES

_ASK = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)
shim.launched_kernels.restype = C.c_char_p
from paper_2605_29346_amd import zg
L, n, out = zg.lib(), C.c_size_t(), []
for rows, k, classes, pad, t, count in json.loads(sys.argv[2]):
    b = zg.LossGradArgs(rows=rows, in_=k, out=classes, dtype=t, label_dtype=zg.I64, d_A=1 << 56, ld_A=k + pad, d_W=2 << 56, ld_W=k + pad, d_labels=3 << 56, d_lse=4 << 56, d_dA=5 << 56, ld_dA=k, d_dW=6 << 56, ld_dW=k,
                        d_dbias=7 << 56, d_rows=(8 << 56) if count else None)
    assert L.zg_linear_cross_entropy_backward_workspace(C.byref(b), C.byref(n)) == 0, L.zg_last_error()
    assert L.zg_linear_cross_entropy_backward(C.byref(b), 9 << 56, n.value, None) == 0, L.zg_last_error()
    out.append(shim.launched_kernels().decode().split())
print(json.dumps(out))
"""
TYPE = {torch.float32: 2, torch.float16: 3, torch.bfloat16: 4}


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    shim = tmp_path_factory.mktemp("shim") / "kernel_shim.so"
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(root, "tests", "kernel_shim.cpp"), "-o", str(shim), "-ldl"], check=True)

    def asked(cases):
        run = subprocess.run([sys.executable, "-c", _ASK, str(shim), json.dumps(cases)], cwd=root, timeout=100, capture_output=True, text=True)
        assert run.returncode == 0, run.stderr[-2000:]
        return json.loads(run.stdout)
    return asked


def _of(launched, what):
    return sum(what in name for name in launched)


def test_pieces_of_rows_and_classes(ask):
    for (rows, k, n, pad, kind, steps, pieces), launched in zip(SIZES, ask([(*s[:4], TYPE[s[4]], True) for s in SIZES])):
        assert _of(launched, "k_loss_dz_") == _of(launched, "k_loss_bias") == steps * pieces, (rows, k, n, launched)
        assert _of(launched, "k_row_counts") == 1 and _of(launched, "k_loss_pack") == (steps + 1 if pad == 3 else 0)


@pytest.mark.parametrize("size,pieces", [((16384, 1024, 65536, 0, 4), 4), ((4099, 301, 10007, 1, 3), 1), ((98765, 256, 47, 0, 2), 1), ((65600, 40, 25003, 0, 4), 7), ((2304, 256, 16, 0, 4), 1), ((0, 8, 8, 0, 2), 0)], ids=str)
def test_other_sizes_take_all_rows_at_once(ask, size, pieces):
    launched, = ask([(*size, False)])
    assert _of(launched, "k_loss_dz_") == pieces and _of(launched, "k_row_counts") == 0
