"""Dense operators on the rows of a mini-batch (the last section of include/zg.h): argument marshalling for torch tensors.

`linear`, `dropout` and `rms_norm` with their gradients, and the same as differentiable functions (`Linear`, `DropoutFn`, `RmsNorm`) for
torch's autograd.  Matrices are 2-D CUDA tensors whose rows are contiguous (`stride(1) == 1`, any `stride(0) >= shape[1]`) of float32,
float16 or bfloat16; `rows` is an int32 CUDA tensor with the number of live rows (e.g. `plan.view_counts()[0][h:h + 1]`): the others are
neither read nor written, and take no part in any sum.  Outputs that are not given are allocated (rows beyond `rows` stay
uninitialised).  Work is enqueued on `stream` (default: torch's current one); nothing synchronises."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import NamedTuple, Optional

import torch

from . import zg

_TYPES = {torch.float32: zg.F32, torch.float16: zg.F16, torch.bfloat16: zg.BF16, torch.float8_e4m3fn: zg.F8}
_ACTS = {"none": zg.ACT_NONE, "relu": zg.ACT_RELU, "silu": zg.ACT_SILU, "gelu": zg.ACT_GELU}


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


def _type(t, what):
    try:
        return _TYPES[t]
    except KeyError:
        raise TypeError(f"{what}: {t} is not one of {', '.join(str(k) for k in _TYPES)}") from None


class _Call:
    """One call: checks the tensors, fills the struct, and keeps what lives on another stream than the one it was made on."""

    def __init__(self, like, rows_t, stream):
        if not like.is_cuda:
            raise ValueError("the operators take CUDA tensors")
        self.device = like.device
        self.stream = zg._stream_ptr(stream if stream is not None else torch.cuda.current_stream(self.device))
        self.foreign = None
        if stream is not None and self.stream != torch.cuda.current_stream(self.device).cuda_stream:
            self.foreign = torch.cuda.ExternalStream(self.stream, device=self.device)
        self.made = []
        self.rows_ptr = self.vector(rows_t, "rows", 1, torch.int32)

    def _device(self, t, what):
        if t.device != self.device:
            raise ValueError(f"{what} is on {t.device}, the others on {self.device}")

    def matrix(self, t, what, rows, cols, dtype):
        self._device(t, what)
        if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols or t.dtype != dtype:
            raise ValueError(f"{what} is {list(t.shape)} of {t.dtype}: [{rows}, {cols}] of {dtype} is wanted")
        if t.stride(1) != 1 and cols > 1:
            raise ValueError(f"the rows of {what} are not contiguous")
        ld = t.stride(0) if rows > 1 else cols
        if rows > 1 and ld < cols:
            raise ValueError(f"the rows of {what} overlap")
        return t.data_ptr(), ld

    def vector(self, t, what, n, dtype=torch.float32):
        if t is None:
            return None
        self._device(t, what)
        if t.numel() != n or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{what} is {list(t.shape)} of {t.dtype}: {n} contiguous elements of {dtype} are wanted")
        return t.data_ptr()

    def make(self, shape, dtype):
        t = torch.empty(shape, dtype=dtype, device=self.device)
        self.made.append(t)
        return t

    def drop(self, d, rows):
        if d is None:
            return zg.Drop()
        return zg.Drop(d.p, d.key & 0xFFFFFFFFFFFFFFFF, d.layer & 0xFFFFFFFF, 0, self.vector(d.ids, "the dropout's ids", rows, torch.int32))

    def run(self, name, args, workspace=False):
        L = zg.lib()
        with torch.cuda.device(self.device):
            if workspace:
                need = C.c_size_t()
                zg._check(getattr(L, name + "_workspace")(C.byref(args), C.byref(need)))
                ws = self.make((need.value,), torch.uint8)
                if self.foreign is not None:  # blocks that torch hands out may still be in use by earlier work of the current stream
                    self.foreign.wait_stream(torch.cuda.current_stream(self.device))
                zg._check(getattr(L, name)(C.byref(args), ws.data_ptr(), need.value, self.stream))
            else:
                if self.foreign is not None and self.made:
                    self.foreign.wait_stream(torch.cuda.current_stream(self.device))
                zg._check(getattr(L, name)(C.byref(args), self.stream))
        if self.foreign is not None:
            for t in self.made:
                t.record_stream(self.foreign)


def _act(act):
    if act not in _ACTS:
        raise ValueError(f"act is {act!r}: one of {', '.join(_ACTS)} is wanted")
    return _ACTS[act]


def linear(a, w, *, bias=None, act="none", dropout: Optional[Dropout] = None, residual=None, scale_a=None, scale_w=None, out_dtype=None,
           rows=None, save=False, out=None, preact=None, stream=None):
    """drop(act(a w^T + bias)) + residual.  a: [rows, in], w: [out, in], bias: [out] float32, residual and result: [rows, out] of
    `out_dtype` (default: a's type; bfloat16 for 8-bit operands).  float8_e4m3fn operands may have scales by row (float32 [rows], [out]).
    `save` (or a tensor `preact`) returns (result, a w^T + bias) for `linear_backward`.  `out` may be the residual."""
    c = _Call(a, rows, stream)
    m, n = a.shape[0], w.shape[0]
    kind = out_dtype or (torch.bfloat16 if a.dtype == torch.float8_e4m3fn else a.dtype)
    out = c.make((m, n), kind) if out is None else out
    preact = c.make((m, n), kind) if preact is None and save else preact
    args = zg.LinearArgs(rows=m, d_rows=c.rows_ptr, in_=a.shape[1], out=n, dtype=_type(a.dtype, "a"), out_dtype=_type(kind, "out_dtype"), act=_act(act))
    args.d_A, args.ld_A = c.matrix(a, "a", m, a.shape[1], a.dtype)
    args.d_W, args.ld_W = c.matrix(w, "w", n, a.shape[1], a.dtype)
    args.d_scale_A, args.d_scale_W = c.vector(scale_a, "scale_a", m), c.vector(scale_w, "scale_w", n)
    args.d_bias = c.vector(bias, "bias", n)
    if residual is not None:
        args.d_R, args.ld_R = c.matrix(residual, "residual", m, n, kind)
    args.d_Y, args.ld_Y = c.matrix(out, "out", m, n, kind)
    if preact is not None:
        args.d_Z, args.ld_Z = c.matrix(preact, "preact", m, n, kind)
    args.drop = c.drop(dropout, m)
    c.run("zg_linear", args)
    return (out, preact) if preact is not None else out


def linear_backward(dy, a, w, *, preact=None, act="none", dropout: Optional[Dropout] = None, rows=None, need=(True, True, True), da=None,
                    dw=None, dbias=None, stream=None):
    """Gradients (da, dw, dbias) of `linear` for the gradient dy of its result (that of the residual is dy itself); `need` says which
    are wanted, the others are None.  `preact` is what `linear(save=True)` returned; without an activation it is not needed."""
    c = _Call(dy, rows, stream)
    m, n, k = dy.shape[0], dy.shape[1], w.shape[1]
    da = c.make((m, k), a.dtype) if da is None and need[0] else da
    dw = c.make((n, k), a.dtype) if dw is None and need[1] else dw
    dbias = c.make((n,), torch.float32) if dbias is None and need[2] else dbias
    args = zg.LinearGradArgs(rows=m, d_rows=c.rows_ptr, in_=k, out=n, dtype=_type(a.dtype, "a"), out_dtype=_type(dy.dtype, "dy"), act=_act(act))
    args.d_dY, args.ld_dY = c.matrix(dy, "dy", m, n, dy.dtype)
    if preact is not None:
        args.d_Z, args.ld_Z = c.matrix(preact, "preact", m, n, dy.dtype)
    args.d_A, args.ld_A = c.matrix(a, "a", m, k, a.dtype)
    args.d_W, args.ld_W = c.matrix(w, "w", n, k, a.dtype)
    if da is not None:
        args.d_dA, args.ld_dA = c.matrix(da, "da", m, k, a.dtype)
    if dw is not None:
        args.d_dW, args.ld_dW = c.matrix(dw, "dw", n, k, a.dtype)
    args.d_dbias = c.vector(dbias, "dbias", n)
    args.drop = c.drop(dropout, m)
    c.run("zg_linear_backward", args, workspace=True)
    return da, dw, dbias


def dropout(x, mask: Optional[Dropout], *, residual=None, rows=None, out=None, stream=None):
    """drop(x) + residual; the gradient of x is the same call on the gradient of the result.  `out` may be x or the residual."""
    c = _Call(x, rows, stream)
    m, n = x.shape
    out = c.make((m, n), x.dtype) if out is None else out
    args = zg.DropoutArgs(rows=m, d_rows=c.rows_ptr, cols=n, dtype=_type(x.dtype, "x"))
    args.d_x, args.ld_x = c.matrix(x, "x", m, n, x.dtype)
    if residual is not None:
        args.d_r, args.ld_r = c.matrix(residual, "residual", m, n, x.dtype)
    args.d_y, args.ld_y = c.matrix(out, "out", m, n, x.dtype)
    args.drop = c.drop(mask, m)
    c.run("zg_dropout", args)
    return out


def rms_norm(x, *, gain=None, eps=1e-6, residual=None, dropout: Optional[Dropout] = None, out_dtype=None, rows=None, y=None, h=None,
             rstd=None, scale=None, stream=None) -> NormResult:
    """h = drop(x) + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd gain (gain: float32 [cols]).  y is of `out_dtype` (default: x's
    type); with float8_e4m3fn y holds y / scale, scale float32 [rows] the row's largest |y| / 448.  h is written where a residual or
    dropout makes it differ from x (or where a tensor `h` is given; that may be the residual or x)."""
    c = _Call(x, rows, stream)
    m, n = x.shape
    kind = out_dtype or x.dtype
    y = c.make((m, n), kind) if y is None else y
    h = c.make((m, n), x.dtype) if h is None and (residual is not None or (dropout is not None and dropout.p > 0)) else h
    rstd = c.make((m,), torch.float32) if rstd is None else rstd
    scale = c.make((m,), torch.float32) if scale is None and kind == torch.float8_e4m3fn else scale
    args = zg.NormArgs(rows=m, d_rows=c.rows_ptr, cols=n, dtype=_type(x.dtype, "x"), out_dtype=_type(kind, "out_dtype"), eps=eps)
    args.d_x, args.ld_x = c.matrix(x, "x", m, n, x.dtype)
    if residual is not None:
        args.d_r, args.ld_r = c.matrix(residual, "residual", m, n, x.dtype)
    args.d_gain = c.vector(gain, "gain", n)
    if h is not None:
        args.d_h, args.ld_h = c.matrix(h, "h", m, n, x.dtype)
    args.d_y, args.ld_y = c.matrix(y, "y", m, n, kind)
    args.d_scale, args.d_rstd = c.vector(scale, "scale", m), c.vector(rstd, "rstd", m)
    args.drop = c.drop(dropout, m)
    c.run("zg_rms_norm", args)
    return NormResult(y, h, rstd, scale)


def rms_norm_backward(dy, h, rstd, *, gain=None, dh=None, dropout: Optional[Dropout] = None, rows=None, need_dr=True, need_dgain=True, dx=None,
                      dr=None, dgain=None, stream=None):
    """Gradients (dx, dr, dgain) of `rms_norm` for the gradient dy of its y and dh of its h (None: nothing reaches h from elsewhere).
    dr, the gradient of the residual, is a tensor of its own only with dropout (else dx is both, and None is returned for it)."""
    c = _Call(dy, rows, stream)
    m, n = dy.shape
    dx = c.make((m, n), dy.dtype) if dx is None else dx
    dr = c.make((m, n), dy.dtype) if dr is None and need_dr and dropout is not None and dropout.p > 0 else dr
    dgain = c.make((n,), torch.float32) if dgain is None and need_dgain else dgain
    args = zg.NormGradArgs(rows=m, d_rows=c.rows_ptr, cols=n, dtype=_type(dy.dtype, "dy"))
    args.d_dy, args.ld_dy = c.matrix(dy, "dy", m, n, dy.dtype)
    args.d_h, args.ld_h = c.matrix(h, "h", m, n, dy.dtype)
    args.d_rstd, args.d_gain = c.vector(rstd, "rstd", m), c.vector(gain, "gain", n)
    if dh is not None:
        args.d_dh, args.ld_dh = c.matrix(dh, "dh", m, n, dy.dtype)
    args.d_dx, args.ld_dx = c.matrix(dx, "dx", m, n, dy.dtype)
    if dr is not None:
        args.d_dr, args.ld_dr = c.matrix(dr, "dr", m, n, dy.dtype)
    args.d_dgain = c.vector(dgain, "dgain", n)
    args.drop = c.drop(dropout, m)
    c.run("zg_rms_norm_backward", args, workspace=True)
    return dx, dr, dgain
