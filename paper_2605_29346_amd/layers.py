"""Dense operators on the rows of a mini-batch (a section of include/zg.h): argument marshalling for torch tensors.

`linear`, `dropout` and `rms_norm` with their gradients (`paper_2605_29346_amd.train` puts them together).  Matrices are 2-D CUDA tensors whose rows are contiguous (`stride(1) == 1`, any `stride(0) >= shape[1]`) of float32,
float16 or bfloat16; `rows` is an int32 CUDA tensor with the number of live rows (e.g. `plan.view_counts()[0][h:h + 1]`): the others are
neither read nor written, and take no part in any sum.  Outputs that are not given are allocated (rows beyond `rows` stay
uninitialised); one that lies on what the call reads is refused, unless it is named below as one that may.  Work is enqueued on `stream` (default: torch's current one; what another stream is to read has to be there when it gets to
it); nothing synchronises.  Autograd does not see the calls: operands that require a gradient are refused where one would be recorded."""
from __future__ import annotations

import ctypes as C
import struct
from dataclasses import dataclass
from typing import NamedTuple, Optional

import torch

from . import zg

_TYPES = {torch.float32: zg.F32, torch.float16: zg.F16, torch.bfloat16: zg.BF16, torch.float8_e4m3fn: zg.F8}
_ACTS = {"none": zg.ACT_NONE, "relu": zg.ACT_RELU, "silu": zg.ACT_SILU, "gelu": zg.ACT_GELU}
_F32, _I32 = torch.float32, torch.int32


@dataclass
class Dropout:
    """A mask of a layer: probability, key of the step, number of the layer, and (optional) int32 ids of the rows, e.g. the plan's
    vertex ids `view_S()`.  Equal masks are equal functions of these: the backward pass takes the same object."""
    p: float
    key: int
    layer: int = 0
    ids: Optional[torch.Tensor] = None


class NormResult(NamedTuple):
    y: torch.Tensor
    h: Optional[torch.Tensor]  # drop(x) + residual; None where that is x itself
    rstd: torch.Tensor
    scale: Optional[torch.Tensor]  # of an 8-bit y


# The structs of include/zg.h as one pack() each (zg.LinearArgs and so on are the same by field): a call of a few rows takes the GPU less
# than filling a ctypes structure field by field takes the host.
_DROP = "dQIIq"
_PACK = {"zg_linear": "@qq6i13q" + _DROP, "zg_linear_backward": "@qq6i13q" + _DROP, "zg_dropout": "@qq2i6q" + _DROP,
         "zg_rms_norm": "@qq3if11q" + _DROP, "zg_rms_norm_backward": "@qq2i13q" + _DROP}
_pack = {name: struct.Struct(f).pack for name, f in _PACK.items()}
_entries: dict = {}


def _entry(name):
    """The library's function, taking the packed struct."""
    f = _entries.get(name)
    if f is None:
        args = [C.c_char_p]
        if name.endswith("_workspace"):
            args.append(C.POINTER(C.c_size_t))
        elif name.endswith("_backward"):
            args += [C.c_void_p, C.c_size_t, C.c_void_p]
        else:
            args.append(C.c_void_p)
        f = _entries[name] = C.CFUNCTYPE(C.c_int, *args)((name, zg.lib()))
    return f


def _type(t, what):
    try:
        return _TYPES[t]
    except KeyError:
        raise TypeError(f"{what}: {t} is not one of {', '.join(str(k) for k in _TYPES)}") from None


def _act(act):
    try:
        return _ACTS[act]
    except KeyError:
        raise ValueError(f"act is {act!r}: one of {', '.join(_ACTS)} is wanted") from None


def _matrix(t, what, rows, cols, dtype, device):
    """(address, row stride)"""
    if t.dtype is not dtype or t.shape != (rows, cols) or t.device != device:
        raise ValueError(f"{what} is {list(t.shape)} of {t.dtype} on {t.device}: [{rows}, {cols}] of {dtype} on {device} is wanted")
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"the rows of {what} are not contiguous")
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise ValueError(f"the rows of {what} overlap")
    return t.data_ptr(), ld


def _vector(t, what, n, dtype, device):
    """address, or 0 for None"""
    if t is None:
        return 0
    if t.dtype is not dtype or t.numel() != n or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} is {list(t.shape)} of {t.dtype} on {t.device}: {n} contiguous elements of {dtype} on {device} are wanted")
    return t.data_ptr()


def _out(t, what, m, n, dtype, device, made, like=None):
    """(tensor, address, row stride) of an output: what the caller gave, or a new one"""
    if t is not None:
        return (t, *_matrix(t, what, m, n, dtype, device))
    t = torch.empty_like(like) if like is not None and like.is_contiguous() else torch.empty((m, n), dtype=dtype, device=device)
    made.append(t)
    return t, t.data_ptr(), n


def _out_vector(t, what, n, device, made):
    """(tensor, address) of an output of float32"""
    if t is not None:
        return t, _vector(t, what, n, _F32, device)
    t = torch.empty(n, dtype=_F32, device=device)
    made.append(t)
    return t, t.data_ptr()


_NONE3 = None, 0, 0


def _no_history(*operands):
    """Refuses operands that autograd would want a gradient of: the results have no history, and it would be lost."""
    if torch.is_grad_enabled():
        for t in operands:
            if t is not None and t.requires_grad:
                raise ValueError("an operand requires a gradient, which the operators do not record: call them under torch.no_grad() or on detached tensors, "
                                 "and linear_backward, dropout or rms_norm_backward for the gradients")


def _shape(t, what):
    """([rows, cols], device) of the operand that a call goes by"""
    if not t.is_cuda:
        raise ValueError("the operators take CUDA tensors")
    if t.dim() != 2:
        raise ValueError(f"{what} is {list(t.shape)}: a matrix is wanted")
    return t.shape, t.device


def _mask(d, rows, device):
    if d is None:
        return 0.0, 0, 0, 0, 0
    return d.p, d.key & 0xFFFFFFFFFFFFFFFF, d.layer & 0xFFFFFFFF, 0, _vector(d.ids, "the dropout's ids", rows, _I32, device)


def _run(name, args, device, stream, made=(), workspace=False):
    """Enqueues the call on `stream`.  `made`: tensors that were allocated for it - on torch's current stream, whose earlier work another
    stream has to wait for, and whose memory must not be handed out again before that other stream is done with it."""
    current = torch._C._cuda_getCurrentRawStream(device.index)
    handle = current if stream is None else zg._stream_ptr(stream)
    foreign = None
    if handle != current:
        foreign = torch.cuda.ExternalStream(handle, device=device)
    args = _pack[name](*args)
    if torch._C._cuda_getDevice() != device.index:
        with torch.cuda.device(device):
            return _enqueue(name, args, device, handle, foreign, made, workspace)
    return _enqueue(name, args, device, handle, foreign, made, workspace)


def _enqueue(name, args, device, handle, foreign, made, workspace):
    if workspace:
        need = C.c_size_t()
        status = _entry(name + "_workspace")(args, C.byref(need))
        if status:
            raise zg.ZgError(status)
        ws = torch.empty(need.value, dtype=torch.uint8, device=device)
        made = (*made, ws)
    if foreign is not None and made:
        foreign.wait_stream(torch.cuda.current_stream(device))
    status = _entry(name)(args, ws.data_ptr(), need.value, handle) if workspace else _entry(name)(args, handle)
    if foreign is not None:
        for t in made:
            t.record_stream(foreign)
    if status:
        raise zg.ZgError(status)


def linear(a, w, *, bias=None, act="none", dropout: Optional[Dropout] = None, residual=None, scale_a=None, scale_w=None, out_dtype=None,
           rows=None, save=False, out=None, preact=None, stream=None):
    """drop(act(a w^T + bias)) + residual.  a: [rows, in], w: [out, in], bias: [out] float32, residual and result: [rows, out] of
    `out_dtype` (default: a's type; bfloat16 for 8-bit operands).  float8_e4m3fn operands may have scales by row (float32 [rows], [out]).
    `save` (or a tensor `preact`) returns (result, a w^T + bias) for `linear_backward`.  `out` may be the residual."""
    _no_history(a, w, bias, residual, scale_a, scale_w)
    (m, k), device = _shape(a, "a")
    n, dtype = w.shape[0], a.dtype
    kind = out_dtype or (torch.bfloat16 if dtype == torch.float8_e4m3fn else dtype)
    made = []
    out, y, ld_y = _out(out, "out", m, n, kind, device, made, a if k == n and kind is dtype else None)
    preact, z, ld_z = _out(preact, "preact", m, n, kind, device, made) if save or preact is not None else _NONE3
    _run("zg_linear", (m, _vector(rows, "rows", 1, _I32, device), k, n, _type(dtype, "a"), _type(kind, "out_dtype"), _act(act), 0,
                       *_matrix(a, "a", m, k, dtype, device), _vector(scale_a, "scale_a", m, _F32, device),
                       *_matrix(w, "w", n, k, dtype, device), _vector(scale_w, "scale_w", n, _F32, device), _vector(bias, "bias", n, _F32, device),
                       *(_matrix(residual, "residual", m, n, kind, device) if residual is not None else (0, 0)),
                       y, ld_y, z, ld_z, *_mask(dropout, m, device)), device, stream, made)
    return (out, preact) if preact is not None else out


def linear_backward(dy, a, w, *, preact=None, act="none", dropout: Optional[Dropout] = None, rows=None, need=(True, True, True), da=None,
                    dw=None, dbias=None, stream=None):
    """Gradients (da, dw, dbias) of `linear` for the gradient dy of its result (that of the residual is dy itself); `need` says which
    are wanted, the others are None.  `preact` is what `linear(save=True)` returned; without an activation it is not needed."""
    _no_history(dy, a, w, preact)
    (m, n), device = _shape(dy, "dy")
    k, dtype, kind = w.shape[1], a.dtype, dy.dtype
    made = []
    da, da_at, ld_da = _out(da, "da", m, k, dtype, device, made) if need[0] or da is not None else _NONE3
    dw, dw_at, ld_dw = _out(dw, "dw", n, k, dtype, device, made) if need[1] or dw is not None else _NONE3
    dbias, db_at = _out_vector(dbias, "dbias", n, device, made) if need[2] or dbias is not None else (None, 0)
    _run("zg_linear_backward", (m, _vector(rows, "rows", 1, _I32, device), k, n, _type(dtype, "a"), _type(kind, "dy"), _act(act), 0,
                                *_matrix(dy, "dy", m, n, kind, device),
                                *(_matrix(preact, "preact", m, n, kind, device) if preact is not None else (0, 0)),
                                *_matrix(a, "a", m, k, dtype, device), *_matrix(w, "w", n, k, dtype, device),
                                da_at, ld_da, dw_at, ld_dw, db_at, *_mask(dropout, m, device)), device, stream, made, workspace=True)
    return da, dw, dbias


def dropout(x, mask: Optional[Dropout], *, residual=None, rows=None, out=None, stream=None):
    """drop(x) + residual; the gradient of x is the same call on the gradient of the result.  `out` may be x or the residual."""
    _no_history(x, residual)
    (m, n), device = _shape(x, "x")
    dtype, made = x.dtype, []
    out, y, ld_y = _out(out, "out", m, n, dtype, device, made, x)
    _run("zg_dropout", (m, _vector(rows, "rows", 1, _I32, device), n, _type(dtype, "x"), *_matrix(x, "x", m, n, dtype, device),
                        *(_matrix(residual, "residual", m, n, dtype, device) if residual is not None else (0, 0)),
                        y, ld_y, *_mask(mask, m, device)), device, stream, made)
    return out


def rms_norm(x, *, gain=None, eps=1e-6, residual=None, dropout: Optional[Dropout] = None, out_dtype=None, rows=None, y=None, h=None,
             rstd=None, scale=None, stream=None) -> NormResult:
    """h = drop(x) + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd gain (gain: float32 [cols]).  y is of `out_dtype` (default: x's
    type); with float8_e4m3fn y holds y / scale, scale float32 [rows] the row's largest |y| / 448.  h is written where a residual or
    dropout makes it differ from x (or where a tensor `h` is given; that may be the residual or x, and so may y be where h is not)."""
    _no_history(x, gain, residual)
    (m, n), device = _shape(x, "x")
    dtype = x.dtype
    kind = out_dtype or dtype
    made = []
    y, y_at, ld_y = _out(y, "y", m, n, kind, device, made, x if kind is dtype else None)
    summed = residual is not None or (dropout is not None and dropout.p > 0)
    h, h_at, ld_h = _out(h, "h", m, n, dtype, device, made, x) if summed or h is not None else _NONE3
    rstd, rstd_at = _out_vector(rstd, "rstd", m, device, made)
    scale, scale_at = _out_vector(scale, "scale", m, device, made) if scale is not None or kind is torch.float8_e4m3fn else (None, 0)
    _run("zg_rms_norm", (m, _vector(rows, "rows", 1, _I32, device), n, _type(dtype, "x"), _type(kind, "out_dtype"), eps,
                         *_matrix(x, "x", m, n, dtype, device),
                         *(_matrix(residual, "residual", m, n, dtype, device) if residual is not None else (0, 0)),
                         _vector(gain, "gain", n, _F32, device), h_at, ld_h, y_at, ld_y, scale_at, rstd_at,
                         *_mask(dropout, m, device)), device, stream, made)
    return NormResult(y, h, rstd, scale)


def rms_norm_backward(dy, h, rstd, *, gain=None, dh=None, dropout: Optional[Dropout] = None, rows=None, need_dr=True, need_dgain=True, dx=None,
                      dr=None, dgain=None, stream=None):
    """Gradients (dx, dr, dgain) of `rms_norm` for the gradient dy of its y and dh of its h (None: nothing reaches h from elsewhere).
    dr, the gradient of the residual, is a tensor of its own only with dropout (else dx is both, and None is returned for it).  dx and dr may
    be dy, h or dh."""
    _no_history(dy, h, rstd, gain, dh)
    (m, n), device = _shape(dy, "dy")
    dtype = dy.dtype
    made = []
    dx, dx_at, ld_dx = _out(dx, "dx", m, n, dtype, device, made, dy)
    two = dr is not None or (need_dr and dropout is not None and dropout.p > 0)
    dr, dr_at, ld_dr = _out(dr, "dr", m, n, dtype, device, made, dy) if two else _NONE3
    dgain, dg_at = _out_vector(dgain, "dgain", n, device, made) if need_dgain or dgain is not None else (None, 0)
    _run("zg_rms_norm_backward", (m, _vector(rows, "rows", 1, _I32, device), n, _type(dtype, "dy"), *_matrix(dy, "dy", m, n, dtype, device),
                                  *_matrix(h, "h", m, n, dtype, device), _vector(rstd, "rstd", m, _F32, device), _vector(gain, "gain", n, _F32, device),
                                  *(_matrix(dh, "dh", m, n, dtype, device) if dh is not None else (0, 0)),
                                  dx_at, ld_dx, dr_at, ld_dr, dg_at, *_mask(dropout, m, device)),
         device, stream, made, workspace=True)
    return dx, dr, dgain
