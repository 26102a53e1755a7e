"""Calls whose outputs lie on what other workgroups still read, or on each other, are refused before anything is launched (the addresses are never
looked at).  What may share a place, and what only lies between another matrix's rows, runs in test_gpu_layers_in_place.py."""
import ctypes as C

import pytest

from paper_2605_29346_amd import zg

AT = {name: (i + 1) << 24 for i, name in enumerate("ABCDEFGHIJ")}
A, B, D, G, H, I, J = (AT[c] for c in "ABDGHIJ")


def _refused(call, args, *rest):
    status = call(C.byref(args), *rest)
    assert status == zg.EINVAL
    assert "lies on" in zg.lib().zg_last_error().decode()


def _with(args, more):
    for k, v in more.items():
        setattr(args, k, v)
    return args


# rows 4, in = out = 8, fp32: a row is 32 bytes, a matrix 128
@pytest.mark.parametrize("more", [
    dict(d_Y=A), dict(d_Y=A + 64), dict(d_Y=A - 32), dict(d_Y=B), dict(d_Y=B + 32, ld_Y=8), dict(d_Z=A, ld_Z=8), dict(d_Z=B, ld_Z=8), dict(d_Z=D, ld_Z=8),
    dict(d_Z=D + 96, ld_Z=8), dict(d_R=D, ld_R=12), dict(d_R=D + 32, ld_R=8), dict(d_R=G, ld_R=8, d_Z=G, ld_Z=8), dict(d_R=G, ld_R=8, d_Z=G + 32, ld_Z=8),
    dict(ld_A=16, ld_Y=16, d_Y=A + 16), dict(ld_A=16, ld_Y=16, d_Y=A - 16), dict(d_bias=D + 32), dict(drop=zg.Drop(p=0.5, d_ids=D)), dict(d_rows=D)])
def test_linear(more):
    _refused(zg.lib().zg_linear, _with(zg.LinearArgs(rows=4, in_=8, out=8, dtype=zg.F32, out_dtype=zg.F32, d_A=A, ld_A=8, d_W=B, ld_W=8, d_Y=D, ld_Y=8), more), None)


@pytest.mark.parametrize("more", [
    dict(d_dA=A), dict(d_dA=B), dict(d_dA=D), dict(d_dA=G), dict(d_dA=A + 32), dict(d_dW=A), dict(d_dW=B), dict(d_dW=D), dict(d_dW=G), dict(d_dW=H), dict(d_dW=H + 96), dict(d_dW=H - 224),
    dict(d_dbias=H), dict(d_dbias=I + 32), dict(d_dbias=A), dict(act=zg.ACT_NONE, d_dA=A)])
def test_linear_backward(more):
    args = zg.LinearGradArgs(rows=4, in_=8, out=8, dtype=zg.F32, out_dtype=zg.F32, act=zg.ACT_SILU, d_dY=A, ld_dY=8, d_Z=B, ld_Z=8, d_A=D, ld_A=8, d_W=G, ld_W=8,
                             d_dA=H, ld_dA=8, d_dW=I, ld_dW=8, d_dbias=J)
    _refused(zg.lib().zg_linear_backward, _with(args, more), 1 << 40, 1 << 40, None)


@pytest.mark.parametrize("more", [dict(d_y=A, ld_y=12), dict(d_y=A + 32), dict(d_y=B, ld_y=16), dict(d_y=B - 32), dict(d_y=A + 4), dict(drop=zg.Drop(p=0.5, d_ids=D))])
def test_dropout(more):
    args = zg.DropoutArgs(rows=4, cols=8, dtype=zg.F32, d_x=A, ld_x=8, d_r=B, ld_r=8, d_y=D, ld_y=8, drop=zg.Drop(p=0.5))
    _refused(zg.lib().zg_dropout, _with(args, more), None)


@pytest.mark.parametrize("more", [
    dict(d_y=G), dict(d_y=G + 32), dict(d_y=A, ld_y=9), dict(d_y=B + 32), dict(out_dtype=zg.BF16, d_y=A), dict(out_dtype=zg.F8, d_y=A, d_scale=I), dict(d_h=A, ld_h=9),
    dict(d_h=B, ld_h=16), dict(d_h=A + 32), dict(d_rstd=D), dict(d_rstd=G + 16), dict(d_rstd=A), dict(d_rstd=H), dict(out_dtype=zg.F8, d_scale=J + 4), dict(out_dtype=zg.F8, d_scale=H)])
def test_norm(more):
    args = zg.NormArgs(rows=4, cols=8, dtype=zg.F32, out_dtype=zg.F32, eps=1e-6, d_x=A, ld_x=8, d_r=B, ld_r=8, d_y=D, ld_y=8, d_h=G, ld_h=8, d_gain=H, d_rstd=J)
    _refused(zg.lib().zg_rms_norm, _with(args, more), None)


@pytest.mark.parametrize("more", [
    dict(d_dx=A, ld_dx=9), dict(d_dx=A + 32), dict(d_dx=B + 32), dict(d_dx=G, ld_dx=16), dict(d_dr=A, ld_dr=9), dict(d_dr=H, drop=zg.Drop(p=0.5)), dict(d_dr=H + 32),
    dict(d_dx=D), dict(d_dgain=H), dict(d_dgain=A), dict(d_dgain=D), dict(d_dx=I)])
def test_norm_backward(more):
    args = zg.NormGradArgs(rows=4, cols=8, dtype=zg.F32, d_dy=A, ld_dy=8, d_h=B, ld_h=8, d_dh=G, ld_dh=8, d_rstd=D, d_gain=I, d_dx=H, ld_dx=8, ld_dr=8, d_dgain=J)
    _refused(zg.lib().zg_rms_norm_backward, _with(args, more), 1 << 40, 1 << 40, None)
