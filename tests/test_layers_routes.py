"""Which kernels the products' rules choose, from the library's own launches: the runtime's launch call is replaced by one that writes their names
down.  No device is needed and nothing is run."""
import json
import os
import re
import subprocess
import sys

import pytest

import layers_routes as S

_ASK = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)
shim.launched_kernels.restype = shim.registered_kernels.restype = C.c_char_p
sys.path.insert(0, "tests")
from paper_2605_29346_amd import zg
import layers_routes as S
L = zg.lib()
KIND = {"f32": (zg.F32, 4), "f16": (zg.F16, 2), "bf16": (zg.BF16, 2), "f8": (zg.F8, 1)}
at = lambda i: i << 44  # (addresses that nobody looks at, far from each other)
out = {"registered": shim.registered_kernels().decode().split("\n"), "forward": [], "backward": []}
def kernels(status):
    assert status == 0, (status, L.zg_last_error())
    return shim.launched_kernels().decode().split()
for t, rows, k, n, pad, epilogue, _ in S.FORWARD:
    a = zg.LinearArgs(rows=rows, in_=k, out=n, dtype=KIND[t][0], d_A=at(1), ld_A=k + pad, d_W=at(2), ld_W=k + pad, d_Y=at(3), ld_Y=n)
    if epilogue == "full":
        a.act, a.d_R, a.ld_R, a.d_Z, a.ld_Z, a.drop = zg.ACT_GELU, at(4), n, at(5), n, zg.Drop(p=0.5)
    for o in ("f32", "f16", "bf16"):
        a.out_dtype = KIND[o][0]
        out["forward"].append(kernels(L.zg_linear(C.byref(a), None)))
for t, o, rows, k, n, pad, *_ in S.BACKWARD:
    a = zg.LinearGradArgs(rows=rows, in_=k, out=n, dtype=KIND[t][0], out_dtype=KIND[o][0], act=zg.ACT_SILU, d_dY=at(1), ld_dY=n + pad, d_Z=at(2), ld_Z=n + pad,
                          d_A=at(3), ld_A=k + pad, d_W=at(4), ld_W=k + pad, d_dA=at(5), ld_dA=k, d_dW=at(6), ld_dW=k, d_dbias=at(7))
    out["backward"].append(kernels(L.zg_linear_backward(C.byref(a), at(8), 1 << 43, None)))
print(json.dumps(out))
"""

MANGLED = {"f32": "f", "f16": "DF16_", "bf16": "DF16b", "f8": "h"}


def _like(kernel, T, O, turned):
    """What a kernel's name begins with.  `turned`: 00, 01 or 11, which operands lie along the rows."""
    t, o = MANGLED[T], MANGLED[O]
    anyhow = "NS0_8Widened8E" if T == "f8" else t
    flags = "".join(f"Lb{b}E" for b in turned)
    if kernel == "few":
        return f"5k_fewI{anyhow}E"
    if kernel.startswith("product"):
        size = kernel.split()[1]
        return f"9k_productI{anyhow}Li{size}ELi{size}E{flags}E"
    if kernel == "long":
        return f"6k_longI{t}{o}{flags}E"
    size = "Li128ELi128ELi3E" if T == "f32" else "Li256ELi128ELi2E"
    return f"8k_chunksI{t}{o}{size}{flags}E"


@pytest.fixture(scope="module")
def asked(tmp_path_factory):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    shim = tmp_path_factory.mktemp("shim") / "kernel_shim.so"
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(root, "tests", "kernel_shim.cpp"), "-o", str(shim), "-ldl"], check=True)
    run = subprocess.run([sys.executable, "-c", _ASK, str(shim)], cwd=root, timeout=100, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-2000:]
    return json.loads(run.stdout)


def _short(names):
    return [n.replace("_ZN2zg12_GLOBAL__N_1", "").replace("_ZN2zg", "") for n in names if n.startswith("_ZN2zg")]


def test_each_size_takes_the_kernel_that_it_is_there_for(asked):
    got = iter(asked["forward"])
    for T, *size, epilogue, kernel in S.FORWARD:
        for O in ("f32", "f16", "bf16"):
            launched = _short(next(got))
            assert len(launched) == 1 and launched[0].startswith(_like(kernel, T, O, "00")), (T, O, size, epilogue, launched)
    for (T, O, *size, dA, dW, parts), launched in zip(S.BACKWARD, asked["backward"]):
        launched = _short(launched)
        expect = (["11k_slope_top"] if T == "f16" and O != "f16" else []) + [f"7k_slopeI{MANGLED[O]}{MANGLED[T]}E", "13k_column_sums", _like(dA, T, T, "01")]
        expect += [_like(dW, T, "f32" if parts else T, "11")] + ["6k_join"] * parts
        assert len(launched) == len(expect) and all(a.startswith(b) for a, b in zip(launched, expect)), (T, O, size, launched, expect)


def test_every_kernel_of_the_products_is_reached(asked):
    every = {n for n in _short(asked["registered"]) if re.match(r"\d+k_(few|product|chunks|long|join|slope|slope_top)(I|E)", n)}
    reached = {n for launched in asked["forward"] + asked["backward"] for n in _short(launched)}
    assert len(every) > 50 and every - reached == set()
