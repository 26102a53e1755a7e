"""CPU-only checks of the loss and the weights' update: struct layouts, refusals before anything touches a device, workspaces, operands that lie on each other or want a gradient."""
import ctypes as C
import os
import struct
import subprocess

import pytest
import torch

from paper_2605_29346_amd import layers, zg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = [("zg_linear_cross_entropy_args", zg.LossArgs, "zg_linear_cross_entropy"), ("zg_linear_cross_entropy_grad_args", zg.LossGradArgs, "zg_linear_cross_entropy_backward"),
         ("zg_orthogonalize_args", zg.OrthogonalizeArgs, "zg_orthogonalize"), ("zg_muon_args", zg.MuonArgs, "zg_muon_step")]


def test_struct_layouts_match_the_header_and_the_packs(tmp_path):
    lines, want = [], []
    for name, mirror, pack in PAIRS:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(mirror))
        for field, _ in mirror._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field.rstrip("_")}));')
            want.append(getattr(mirror, field).offset)
        values = [i + (0.5 if t is C.c_float else 0) for i, (_, t) in enumerate(mirror._fields_)]
        packed = struct.pack(layers._PACK[pack], *values)
        assert len(packed) == C.sizeof(mirror)
        for (field, t), v in zip(mirror._fields_, values):
            assert t.from_buffer_copy(packed, getattr(mirror, field).offset).value == v, (name, field)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "zg.h"\nint main(void){' + "\n".join(lines) + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


AT = {c: (i + 1) << 24 for i, c in enumerate("ABCDEFGHIJKLM")}
A, W, BIAS, LABELS, WEIGHT, LOSS, TOTAL, LSE, EACH, DA, DW, DBIAS, WS = (AT[c] for c in "ABCDEFGHIJKLM")
BIG = 1 << 40


def _loss(**more):
    a = zg.LossArgs(rows=4, in_=8, out=8, dtype=zg.F32, label_dtype=zg.I64, d_A=A, ld_A=8, d_W=W, ld_W=8, d_bias=BIAS, d_labels=LABELS, d_weight=WEIGHT, d_loss=LOSS, d_total=TOTAL, d_lse=LSE,
                    d_row_loss=EACH)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def _grad(**more):
    a = zg.LossGradArgs(rows=4, in_=8, out=8, dtype=zg.F32, label_dtype=zg.I64, d_A=A, ld_A=8, d_W=W, ld_W=8, d_bias=BIAS, d_labels=LABELS, d_weight=WEIGHT, d_lse=LSE, d_total=TOTAL, d_dloss=LOSS,
                        d_dA=DA, ld_dA=8, d_dW=DW, ld_dW=8, d_dbias=DBIAS)
    for k, v in more.items():
        setattr(a, k, v)
    return a


SAME = [dict(rows=-1), dict(rows=1 << 31), dict(in_=0), dict(in_=zg.MAX_WIDTH + 1), dict(out=0), dict(out=zg.MAX_CLASSES + 1), dict(dtype=zg.F8), dict(dtype=zg.I64), dict(label_dtype=zg.F32), dict(label_dtype=9),
        dict(d_A=None), dict(d_W=None), dict(d_labels=None), dict(ld_A=7), dict(ld_W=7), dict(d_A=A + 2), dict(d_W=W + 1), dict(d_bias=BIAS + 2), dict(d_labels=LABELS + 4), dict(label_dtype=zg.I32, d_labels=LABELS + 2),
        dict(d_weight=WEIGHT + 1), dict(d_rows=BIAS + 2), dict(d_lse=None), dict(d_lse=LSE + 2)]


@pytest.mark.parametrize("bad", SAME + [dict(d_loss=None), dict(d_loss=LOSS + 1), dict(d_total=TOTAL + 2), dict(d_row_loss=EACH + 3)])
def test_loss_refuses(bad):
    assert zg.lib().zg_linear_cross_entropy(C.byref(_loss(**bad)), WS, BIG, None) == zg.EINVAL
    assert zg.lib().zg_last_error()


@pytest.mark.parametrize("bad", SAME + [dict(ld_dA=7), dict(ld_dW=7), dict(d_dA=DA + 1), dict(d_dW=DW + 2), dict(d_dbias=DBIAS + 2), dict(d_total=TOTAL + 1), dict(d_dloss=LOSS + 2)])
def test_loss_backward_refuses(bad):
    assert zg.lib().zg_linear_cross_entropy_backward(C.byref(_grad(**bad)), WS, BIG, None) == zg.EINVAL


# fp32: a row of A or W is 32 bytes, four or eight of them; the labels are 32 bytes, vectors over the rows 16
@pytest.mark.parametrize("more", [dict(d_loss=A), dict(d_loss=W + 252), dict(d_loss=LABELS + 28), dict(d_total=LOSS), dict(d_total=BIAS), dict(d_lse=A + 112), dict(d_lse=LABELS), dict(d_lse=WEIGHT + 12), dict(d_lse=LOSS),
                                  dict(d_row_loss=LSE), dict(d_row_loss=LSE + 12), dict(d_row_loss=WEIGHT), dict(d_row_loss=BIAS + 28), dict(d_rows=LSE), dict(d_rows=LOSS)])
def test_loss_outputs_that_lie_on_something(more):
    assert zg.lib().zg_linear_cross_entropy(C.byref(_loss(**more)), WS, BIG, None) == zg.EINVAL
    assert "lies on" in zg.lib().zg_last_error().decode()


@pytest.mark.parametrize("more", [dict(d_dA=A), dict(d_dA=W), dict(d_dA=A + 96), dict(d_dA=LABELS), dict(d_dW=W), dict(d_dW=A), dict(d_dW=DA), dict(d_dW=DA + 96), dict(d_dW=LSE - 240), dict(d_dbias=DW), dict(d_dbias=BIAS),
                                  dict(d_dbias=LSE + 12), dict(d_dbias=DA), dict(d_dA=TOTAL), dict(d_dbias=LOSS - 28), dict(d_rows=DW + 64)])
def test_loss_gradients_that_lie_on_something(more):
    assert zg.lib().zg_linear_cross_entropy_backward(C.byref(_grad(**more)), WS, BIG, None) == zg.EINVAL
    assert "lies on" in zg.lib().zg_last_error().decode()


K = (C.c_float * 96)(*([3.4445, -4.7750, 2.0315] * 32))


def _orth(**more):
    a = zg.OrthogonalizeArgs(rows=4, cols=8, dtype=zg.F32, out_dtype=zg.F32, steps=5, eps=1e-7, coefficients=C.addressof(K), d_G=A, ld_G=8, d_O=W, ld_O=8)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def _muon(**more):
    a = zg.MuonArgs(rows=4, cols=8, dtype=zg.F32, grad_dtype=zg.F32, steps=5, nesterov=1, lr=0.1, momentum=0.9, decay=0.0, scale=1.0, eps=1e-7, coefficients=C.addressof(K), d_G=A, ld_G=8, d_M=BIAS, ld_M=8,
                    d_W=W, ld_W=8)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def _triples(*values):
    k = (C.c_float * 96)(*(list(values) * 32))
    _triples.kept.append(k)
    return C.addressof(k)


_triples.kept = []
BOTH = [dict(rows=0), dict(rows=-1), dict(cols=0), dict(rows=zg.MAX_WIDTH + 1), dict(cols=zg.MAX_WIDTH + 1), dict(dtype=zg.F8), dict(dtype=zg.I32), dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(coefficients=None), dict(d_G=None), dict(ld_G=7), dict(d_G=A + 2), dict(coefficients=_triples(float("nan"), 0, 0)), dict(coefficients=_triples(1, float("inf"), 0)),
        dict(coefficients=_triples(100.0, 0, 0)), dict(coefficients=_triples(3.0, 3.0, 3.0)), dict(coefficients=_triples(1, 0, 2e6))]


@pytest.mark.parametrize("bad", BOTH + [dict(out_dtype=zg.F8), dict(d_O=None), dict(ld_O=7), dict(d_O=W + 1)])
def test_orthogonalize_refuses(bad):
    assert zg.lib().zg_orthogonalize(C.byref(_orth(**bad)), WS, BIG, None) == zg.EINVAL
    assert zg.lib().zg_last_error()


@pytest.mark.parametrize("bad", BOTH + [dict(grad_dtype=zg.F8), dict(d_W=None), dict(d_M=None), dict(ld_M=7), dict(ld_W=7), dict(d_M=BIAS + 2), dict(lr=float("nan")), dict(momentum=float("inf")), dict(decay=float("nan")),
                                        dict(scale=float("inf"))])
def test_muon_refuses(bad):
    assert zg.lib().zg_muon_step(C.byref(_muon(**bad)), WS, BIG, None) == zg.EINVAL


@pytest.mark.parametrize("call,args", [("zg_orthogonalize", _orth(d_O=A + 32)), ("zg_orthogonalize", _orth(d_O=A, ld_O=12)), ("zg_orthogonalize", _orth(d_O=A, out_dtype=zg.BF16)), ("zg_muon_step", _muon(d_M=A)),
                                       ("zg_muon_step", _muon(d_W=A)), ("zg_muon_step", _muon(d_M=W)), ("zg_muon_step", _muon(d_W=BIAS + 96)), ("zg_muon_step", _muon(d_W=A - 96))])
def test_matrices_that_lie_on_each_other(call, args):
    assert getattr(zg.lib(), call)(C.byref(args), WS, BIG, None) == zg.EINVAL
    assert "lies on" in zg.lib().zg_last_error().decode()


@pytest.mark.parametrize("call,args", [("zg_linear_cross_entropy", _loss()), ("zg_linear_cross_entropy_backward", _grad()), ("zg_orthogonalize", _orth()), ("zg_muon_step", _muon())])
def test_workspaces_and_null_structs(call, args):
    L, n = zg.lib(), C.c_size_t()
    run, ask = getattr(L, call), getattr(L, call + "_workspace")
    assert ask(C.byref(args), C.byref(n)) == zg.OK and n.value > 0
    assert run(C.byref(args), WS, n.value - 1, None) == zg.ENOMEM
    assert run(C.byref(args), None, n.value, None) == zg.EINVAL
    assert run(C.byref(args), WS + 64, n.value, None) == zg.EINVAL
    assert ask(C.byref(args), None) == zg.EINVAL and ask(None, C.byref(n)) == zg.EINVAL and run(None, WS, n.value, None) == zg.EINVAL


def test_workspaces_stay_below_the_logits():
    L, n = zg.lib(), C.c_size_t()
    rows, k, classes = 65536, 1024, 131072
    logits = rows * classes * 2
    a = _loss(rows=rows, in_=k, out=classes, dtype=zg.BF16, ld_A=k, ld_W=k, d_W=1 << 44, d_labels=1 << 45, d_weight=None)
    assert L.zg_linear_cross_entropy_workspace(C.byref(a), C.byref(n)) == zg.OK and n.value < logits / 15
    b = _grad(rows=rows, in_=k, out=classes, dtype=zg.BF16, ld_A=k, ld_W=k, d_W=1 << 44, d_labels=1 << 45, d_weight=None)
    assert L.zg_linear_cross_entropy_backward_workspace(C.byref(b), C.byref(n)) == zg.OK and n.value < logits / 7


X, V, Y = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, dtype=torch.int64)
CALLS = {
    "linear_cross_entropy": (lambda **t: layers.linear_cross_entropy(t.pop("a", X), t.pop("w", X), Y, **t), {"a": X, "w": X, "bias": V, "weight": V}),
    "linear_cross_entropy_backward": (lambda **t: layers.linear_cross_entropy_backward(t.pop("a", X), t.pop("w", X), Y, t.pop("lse", V), **t), {"a": X, "w": X, "lse": V, "bias": V, "weight": V, "total": V, "dloss": V}),
    "orthogonalize": (lambda **t: layers.orthogonalize(t.pop("g", X), **t), {"g": X}),
    "muon_step": (lambda **t: layers.muon_step(t.pop("w", X), t.pop("m", X), t.pop("g", X), lr=0.1, **t), {"w": X, "m": X, "g": X}),
}


@pytest.mark.parametrize("name,operand", [(name, operand) for name, (_, operands) in CALLS.items() for operand in operands])
def test_an_operand_that_wants_a_gradient_is_refused(name, operand):
    call, operands = CALLS[name]
    wants = operands[operand].clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        call(**{operand: wants})
    with pytest.raises(ValueError, match="CUDA"):
        call(**{operand: wants.detach()})
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
        call(**{operand: wants})


@pytest.mark.parametrize("bad", [dict(steps=0), dict(steps=33), dict(steps=2.0), dict(coefficients=(1.0, 2.0)), dict(coefficients=()), dict(coefficients=[(1.0, 0.0, 0.0)], steps=2), dict(coefficients=[(1.0, 0.0)], steps=1)])
def test_coefficients_are_checked(bad):
    with pytest.raises(ValueError, match="wanted"):
        layers._steps(bad.get("coefficients", layers.NEWTON_SCHULZ), bad.get("steps", 5))


def test_coefficients_for_each_step():
    k = layers._steps([(1.0, 2.0, 3.0), (4.0, 5.0, 6.0)], 2)
    assert list(k) == [1, 2, 3, 4, 5, 6] and list(layers._steps((1, 2, 3), 2)) == [1, 2, 3, 1, 2, 3]
