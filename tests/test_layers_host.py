"""CPU-only checks of the dense operators: struct layouts, the mask's definition, refusals before anything touches a device."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import layers, zg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header(tmp_path):
    pairs = [("zg_drop", zg.Drop), ("zg_linear_args", zg.LinearArgs), ("zg_linear_grad_args", zg.LinearGradArgs), ("zg_dropout_args", zg.DropoutArgs),
             ("zg_norm_args", zg.NormArgs), ("zg_norm_grad_args", zg.NormGradArgs)]
    lines, want = [], []
    for name, mirror in pairs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(mirror))
        for field, _ in mirror._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field.rstrip("_")}));')
            want.append(getattr(mirror, field).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include "zg.h"\nint main(void){' + "\n".join(lines) + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def test_the_masks_generator_gives_the_published_words():
    n = 0
    for line in open(os.path.join(ROOT, "tests", "golden", "philox4x32_10_kat.txt")):
        words = [int(x, 16) for x in line.split("#")[0].split()[-10:] if all(ch in "0123456789abcdefABCDEFx" for ch in x)]
        if len(words) < 10:
            continue
        got = [int(x[0]) for x in R.philox([np.array([v]) for v in words[:4]], words[4:6])]
        assert got == words[6:10]
        n += 1
    assert n >= 3


def test_the_mask_keeps_its_share_and_differs_by_key_layer_and_row():
    p, rows, cols = 0.25, 2000, 96
    k = R.kept(p, 77, 3, range(rows), cols).numpy()
    n = k.size
    assert abs(k.mean() - (1 - p)) < 5 * (p * (1 - p) / n) ** 0.5
    assert np.abs(k.mean(0) - (1 - p)).max() < 5 * (p * (1 - p) / rows) ** 0.5
    for other in (R.kept(p, 78, 3, range(rows), cols), R.kept(p, 77, 4, range(rows), cols), R.kept(p, 77, 3, range(rows, 2 * rows), cols)):
        same = (other.numpy() == k).mean()
        expect = p * p + (1 - p) ** 2
        assert abs(same - expect) < 5 * (expect * (1 - expect) / n) ** 0.5


FAKE = 1 << 20  # an address that no refused call looks at


def _linear(**more):
    a = zg.LinearArgs(rows=4, in_=8, out=8, dtype=zg.F32, out_dtype=zg.F32, d_A=FAKE, ld_A=8, d_W=2 * FAKE, ld_W=8, d_Y=3 * FAKE, ld_Y=8)
    for k, v in more.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(in_=0), dict(out=0), dict(in_=zg.MAX_WIDTH + 1), dict(dtype=zg.I32), dict(out_dtype=zg.F8), dict(out_dtype=9),
    dict(act=4), dict(act=-1), dict(d_A=None), dict(d_W=None), dict(d_Y=None), dict(ld_A=7), dict(ld_W=7), dict(ld_Y=7), dict(d_A=FAKE + 2), dict(d_Y=FAKE),
    dict(d_Z=3 * FAKE, ld_Z=8), dict(d_Z=5 * FAKE, ld_Z=7), dict(d_R=5 * FAKE, ld_R=7), dict(d_R=5 * FAKE, ld_R=8, d_Z=5 * FAKE, ld_Z=8), dict(d_scale_A=FAKE),
    dict(d_scale_W=FAKE), dict(d_bias=FAKE + 1), dict(d_rows=FAKE + 2), dict(drop=zg.Drop(p=-0.1)), dict(drop=zg.Drop(p=1.1)),
    dict(drop=zg.Drop(p=float("nan"))), dict(drop=zg.Drop(p=0.5, d_ids=FAKE + 1))])
def test_linear_refuses(bad):
    assert zg.lib().zg_linear(C.byref(_linear(**bad)), None) == zg.EINVAL
    assert zg.lib().zg_last_error()


def test_null_structs_are_refused():
    L, n = zg.lib(), C.c_size_t()
    assert L.zg_linear(None, None) == zg.EINVAL and L.zg_dropout(None, None) == zg.EINVAL and L.zg_rms_norm(None, None) == zg.EINVAL
    assert L.zg_linear_backward(None, None, 0, None) == zg.EINVAL and L.zg_rms_norm_backward(None, None, 0, None) == zg.EINVAL
    assert L.zg_linear_backward_workspace(None, C.byref(n)) == zg.EINVAL and L.zg_rms_norm_backward_workspace(None, C.byref(n)) == zg.EINVAL


def _grad(**more):
    a = zg.LinearGradArgs(rows=4, in_=8, out=8, dtype=zg.F32, out_dtype=zg.F32, act=zg.ACT_SILU, d_dY=FAKE, ld_dY=8, d_Z=2 * FAKE, ld_Z=8, d_A=3 * FAKE,
                          ld_A=8, d_W=4 * FAKE, ld_W=8, d_dA=5 * FAKE, ld_dA=8, d_dW=6 * FAKE, ld_dW=8, d_dbias=7 * FAKE)
    for k, v in more.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(in_=0), dict(out=zg.MAX_WIDTH + 1), dict(dtype=zg.F8), dict(out_dtype=zg.F8), dict(act=7), dict(d_dY=None), dict(d_Z=None),
    dict(d_A=None), dict(d_W=None), dict(ld_dY=7), dict(ld_Z=7), dict(ld_A=7), dict(ld_W=7), dict(ld_dA=7), dict(ld_dW=7), dict(d_dbias=FAKE + 2),
    dict(d_rows=FAKE + 1), dict(drop=zg.Drop(p=2.0))])
def test_linear_backward_refuses(bad):
    assert zg.lib().zg_linear_backward(C.byref(_grad(**bad)), FAKE, 1 << 40, None) == zg.EINVAL


def test_workspaces_are_checked():
    L, n = zg.lib(), C.c_size_t()
    assert L.zg_linear_backward_workspace(C.byref(_grad()), C.byref(n)) == zg.OK and n.value > 0
    assert L.zg_linear_backward(C.byref(_grad()), FAKE, n.value - 1, None) == zg.ENOMEM
    assert L.zg_linear_backward(C.byref(_grad()), None, n.value, None) == zg.EINVAL
    assert L.zg_linear_backward(C.byref(_grad()), FAKE + 64, n.value, None) == zg.EINVAL
    assert L.zg_linear_backward_workspace(C.byref(_grad()), None) == zg.EINVAL
    assert L.zg_rms_norm_backward_workspace(C.byref(_norm_grad()), C.byref(n)) == zg.OK and n.value > 0
    assert L.zg_rms_norm_backward(C.byref(_norm_grad()), FAKE, n.value - 1, None) == zg.ENOMEM
    assert L.zg_rms_norm_backward_workspace(C.byref(_norm_grad(d_dgain=None)), C.byref(n)) == zg.OK and n.value == 0


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=0), dict(dtype=zg.F8), dict(d_x=None), dict(d_y=None), dict(ld_x=7), dict(ld_y=7),
                                 dict(d_r=FAKE, ld_r=7), dict(d_x=FAKE + 1), dict(drop=zg.Drop(p=1.5))])
def test_dropout_refuses(bad):
    a = zg.DropoutArgs(rows=4, cols=8, dtype=zg.F32, d_x=FAKE, ld_x=8, d_y=2 * FAKE, ld_y=8, drop=zg.Drop(p=0.5))
    for k, v in bad.items():
        setattr(a, k, v)
    assert zg.lib().zg_dropout(C.byref(a), None) == zg.EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=zg.MAX_NORM_WIDTH + 1), dict(dtype=zg.F8), dict(out_dtype=zg.I64), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(d_x=None), dict(d_y=None), dict(ld_x=7), dict(d_r=FAKE, ld_r=3), dict(d_h=FAKE, ld_h=3), dict(out_dtype=zg.F8),
                                 dict(d_gain=FAKE + 2), dict(d_rstd=FAKE + 1), dict(drop=zg.Drop(p=-1.0))])
def test_norm_refuses(bad):
    a = zg.NormArgs(rows=4, cols=8, dtype=zg.F32, out_dtype=zg.F32, eps=1e-6, d_x=FAKE, ld_x=8, d_y=2 * FAKE, ld_y=8)
    for k, v in bad.items():
        setattr(a, k, v)
    assert zg.lib().zg_rms_norm(C.byref(a), None) == zg.EINVAL


def _norm_grad(**more):
    a = zg.NormGradArgs(rows=4, cols=8, dtype=zg.F32, d_dy=FAKE, ld_dy=8, d_h=2 * FAKE, ld_h=8, d_rstd=3 * FAKE, d_dx=4 * FAKE, ld_dx=8, d_dgain=5 * FAKE)
    for k, v in more.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=0), dict(dtype=zg.F8), dict(d_dy=None), dict(d_h=None), dict(d_rstd=None), dict(d_dx=None),
                                 dict(ld_dy=7), dict(ld_h=7), dict(ld_dx=7), dict(d_dh=FAKE, ld_dh=7), dict(d_dr=FAKE, ld_dr=7), dict(d_gain=FAKE + 1)])
def test_norm_backward_refuses(bad):
    assert zg.lib().zg_rms_norm_backward(C.byref(_norm_grad(**bad)), FAKE, 1 << 40, None) == zg.EINVAL


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    for call in (lambda: layers.linear(x, x), lambda: layers.dropout(x, None), lambda: layers.rms_norm(x), lambda: layers.linear_backward(x, x, x),
                 lambda: layers.rms_norm_backward(x, x, x[:, 0])):
        with pytest.raises(ValueError):
            call()


def test_no_rows_is_no_work():
    # nothing is launched, so this needs no device
    a = _linear(rows=0)
    assert zg.lib().zg_linear(C.byref(a), None) == zg.OK
    assert zg.lib().zg_dropout(C.byref(zg.DropoutArgs(rows=0, cols=8, dtype=zg.F32)), None) == zg.OK
    assert zg.lib().zg_rms_norm(C.byref(zg.NormArgs(rows=0, cols=8, dtype=zg.F32, out_dtype=zg.F32)), None) == zg.OK


def test_the_packed_structs_are_the_same_field_by_field():
    import struct
    for name, mirror in (("zg_linear", zg.LinearArgs), ("zg_linear_backward", zg.LinearGradArgs), ("zg_dropout", zg.DropoutArgs),
                         ("zg_rms_norm", zg.NormArgs), ("zg_rms_norm_backward", zg.NormGradArgs)):
        flat = [(f, t, getattr(mirror, f).offset) for f, t in mirror._fields_ if f != "drop"]
        flat += [(f, t, mirror.drop.offset + getattr(zg.Drop, f).offset) for f, t in zg.Drop._fields_]
        values = [i + (0.5 if t in (C.c_double, C.c_float) else 0) for i, (_, t, _) in enumerate(flat)]
        packed = struct.pack(layers._PACK[name], *values)
        assert len(packed) == C.sizeof(mirror)
        for (field, t, at), v in zip(flat, values):
            assert t.from_buffer_copy(packed, at).value == v, (name, field)
