"""8-bit activation checkpoints and the norms, on torch tensors.

The calls of ``include/ampq.h`` (``ampq_ckpt_*``, ``ampq_norm_*``) for tensors:
shapes, pitches and dtypes are read off the tensors, outputs and workspaces come
from torch's caching allocator, and everything runs on torch's current stream of
the tensors' device.  ``linear``, ``layer_norm`` and ``rms_norm`` are the same as
differentiable functions that keep their input in 8 bits for the backward pass;
``hooks.Calibrator(checkpoint=...)`` runs a model's layers through them.

Operands are float32 or bfloat16.  A tensor of more than two dimensions is a
matrix of its last dimension; rows may lie further apart than they are long (a
slice of a wider tensor is read in place), anything else is made contiguous.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as ampq
from .binding import AmpqError

_CODE = {torch.float32: ampq.F32, torch.bfloat16: ampq.BF16}


class Packed:
    """A checkpoint: ``codes`` [rows, columns rounded up to whole groups of 32] and
    ``scales`` [rows, groups], both uint8 on the device, of a matrix of ``cols``
    columns in format ``fmt`` (``FMT_E4M3`` or ``FMT_E5M2``)."""

    __slots__ = ("codes", "scales", "cols", "fmt")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int, fmt: int):
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2 or scales.dim() != 2:
            raise TypeError("codes and scales are uint8 matrices")
        if not codes.is_cuda or codes.device != scales.device:
            raise ValueError("codes and scales are on one CUDA device")
        groups = -(-cols // ampq.CKPT_GROUP)
        if codes.shape[0] != scales.shape[0] or codes.shape[1] < groups * ampq.CKPT_GROUP or scales.shape[1] < groups:
            raise ValueError("codes %s and scales %s do not hold %d columns" % (tuple(codes.shape), tuple(scales.shape), cols))
        if (codes.shape[1] > 1 and codes.stride(1) != 1) or (scales.shape[1] > 1 and scales.stride(1) != 1):
            raise ValueError("codes and scales lie contiguously within a row")
        self.codes, self.scales, self.cols, self.fmt = codes, scales, cols, fmt

    @property
    def rows(self) -> int:
        return self.codes.shape[0]

    @property
    def device(self):
        return self.codes.device

    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()


def _check(rc: int, what: str):
    if rc:
        raise AmpqError(rc, what)


def _where(t: torch.Tensor):
    """(device index, current stream's handle) of a tensor."""
    if not t.is_cuda:
        raise ValueError("tensors are on a CUDA device, got %s" % t.device)
    return t.device.index, torch._C._cuda_getCurrentRawStream(t.device.index)


def _code(t: torch.Tensor) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError("operands are float32 or bfloat16, got %s" % t.dtype)
    return code


def _pitch(t: torch.Tensor) -> int:
    """Elements between two rows of a matrix with contiguous rows."""
    return t.stride(0) if t.shape[0] > 1 and t.shape[1] > 0 else t.shape[1]


def _matrix(t: torch.Tensor) -> torch.Tensor:
    """t as rows of its last dimension, without a copy where the layout allows it."""
    if t.dim() == 0:
        raise ValueError("operands have at least one dimension")
    m = t
    if t.dim() != 2:
        rows = 1
        for d in t.shape[:-1]:
            rows *= d
        m = t.reshape(rows, t.shape[-1])  # a view where it can be one
    if (m.shape[1] > 1 and m.stride(1) != 1) or (m.shape[0] > 1 and m.stride(0) < m.shape[1]):
        m = m.contiguous()
    return m


def _same_device(first: torch.Tensor, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("operands are on one device, got %s and %s" % (first.device, t.device))


def _new_packed(rows: int, cols: int, fmt: int, device) -> Packed:
    groups = -(-cols // ampq.CKPT_GROUP)
    codes = torch.empty(rows, groups * ampq.CKPT_GROUP, dtype=torch.uint8, device=device)
    scales = torch.empty(rows, groups, dtype=torch.uint8, device=device)
    return Packed(codes, scales, cols, fmt)


def _packed_args(p: Packed):
    return p.codes.data_ptr(), _pitch(p.codes), p.scales.data_ptr(), _pitch(p.scales)


def _param(t, cols: int, like=None):
    """A parameter vector of `cols` elements, contiguous."""
    if t is None:
        return None
    if t.numel() != cols:
        raise ValueError("a norm over %d columns has parameters of that many elements, got %s" % (cols, tuple(t.shape)))
    if like is not None and like.dtype != t.dtype:
        raise TypeError("weight and bias are of one type, got %s and %s" % (like.dtype, t.dtype))
    return t.reshape(-1).contiguous()


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def pack(x: torch.Tensor, fmt: int = ampq.FMT_E4M3) -> Packed:
    """The 8-bit checkpoint of x."""
    m = _matrix(x)
    device, stream = _where(m)
    p = _new_packed(m.shape[0], m.shape[1], fmt, m.device)
    _check(ampq.lib().ampq_ckpt_pack(device, stream, _code(m), fmt, m.data_ptr(), m.shape[0], m.shape[1], _pitch(m), *_packed_args(p)),
           "ampq_ckpt_pack")
    return p


def unpack(p: Packed, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values a checkpoint stands for, [rows, cols]; exact in either type."""
    out = torch.empty(p.rows, p.cols, dtype=dtype, device=p.device)
    device, stream = _where(out)
    _check(ampq.lib().ampq_ckpt_unpack(device, stream, _code(out), p.fmt, *_packed_args(p), p.rows, p.cols, out.data_ptr(), _pitch(out)),
           "ampq_ckpt_unpack")
    return out


def weight_grad(p: Packed, gy: torch.Tensor, samples: int = 1, bias: bool = False):
    """Weight gradients of a linear layer from the checkpoint of its input and the
    gradient of its output, one per sample: the rows are ``samples`` equal runs.
    Returns (gw [samples, outs, cols], gb [samples, outs] or None) in gy's type."""
    g = _matrix(gy)
    _same_device(p.codes, g)
    if samples < 1 or g.shape[0] != p.rows or p.rows % samples:
        raise ValueError("%d gradient rows, %d checkpoint rows, %d samples" % (g.shape[0], p.rows, samples))
    device, stream = _where(g)
    rows, outs, code = p.rows // samples, g.shape[1], _code(g)
    L = ampq.lib()
    gw = torch.empty(samples, outs, p.cols, dtype=g.dtype, device=g.device)
    gb = torch.empty(samples, outs, dtype=g.dtype, device=g.device) if bias else None
    need = C.c_longlong()
    _check(L.ampq_ckpt_weight_grad_workspace(device, code, g.data_ptr(), _pitch(g), samples, rows, p.cols, outs, 1 if bias else 0,
                                             C.byref(need)), "ampq_ckpt_weight_grad_workspace")
    ws = torch.empty(need.value, dtype=torch.uint8, device=g.device) if need.value else None
    _check(L.ampq_ckpt_weight_grad(device, stream, code, p.fmt, g.data_ptr(), _pitch(g), *_packed_args(p), samples, rows, p.cols, outs,
                                   gw.data_ptr(), _ptr(gb), _ptr(ws), need.value), "ampq_ckpt_weight_grad")
    return gw, gb


def norm_forward(x: torch.Tensor, weight, bias, eps: float, kind: int = ampq.NORM_LAYER, fmt: int = ampq.FMT_BASE):
    """Layer norm or RMS norm over the last dimension.  Returns (y, mean, rstd, p):
    mean is None for an RMS norm, p the checkpoint of x or None for ``FMT_BASE``."""
    m = _matrix(x)
    _same_device(m, weight, bias)
    device, stream = _where(m)
    rows, cols = m.shape
    weight = _param(weight, cols)
    bias = _param(bias, cols, weight)
    first = weight if weight is not None else bias
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    mean = torch.empty(rows, dtype=torch.float32, device=x.device) if kind == ampq.NORM_LAYER else None
    p = _new_packed(rows, cols, fmt, x.device) if fmt != ampq.FMT_BASE else None
    _check(ampq.lib().ampq_norm_forward(device, stream, kind, _code(m), _code(first) if first is not None else _code(m), fmt, m.data_ptr(),
                                        _pitch(m), rows, cols, _ptr(weight), _ptr(bias), eps, y.data_ptr(), cols, _ptr(mean),
                                        rstd.data_ptr(), *(_packed_args(p) if p is not None else (0, 0, 0, 0))), "ampq_norm_forward")
    return y, mean, rstd, p


def norm_backward(gy: torch.Tensor, x, mean, rstd: torch.Tensor, weight, kind: int = ampq.NORM_LAYER, bias: bool = True):
    """Backward pass of ``norm_forward``; x is the input or its checkpoint.  Returns
    (gx, gw, gb): gw is None without a weight, gb unless a layer norm with a bias."""
    g = _matrix(gy)
    rows, cols = g.shape
    kept = isinstance(x, Packed)
    if not kept:
        x = _matrix(x)
    _same_device(g, x.codes if kept else x, mean, rstd, weight)
    if (x.rows, x.cols) != (rows, cols) if kept else tuple(x.shape) != (rows, cols):
        raise ValueError("the input does not have the gradient's %d rows of %d columns" % (rows, cols))
    if not kept and x.dtype != g.dtype:
        raise TypeError("input and gradient are of one type, got %s and %s" % (x.dtype, g.dtype))
    for t in (rstd, mean) if kind == ampq.NORM_LAYER else (rstd,):
        if t is None or t.dtype != torch.float32 or t.numel() != rows or not t.is_contiguous():
            raise ValueError("mean and rstd are as norm_forward returned them")
    device, stream = _where(g)
    weight = _param(weight, cols)
    gx = torch.empty(gy.shape, dtype=g.dtype, device=g.device)
    pdtype = weight.dtype if weight is not None else g.dtype
    bias = bias and kind == ampq.NORM_LAYER
    sums = weight is not None or bias
    gw = torch.empty(cols, dtype=pdtype, device=g.device) if sums else None
    gb = torch.empty(cols, dtype=pdtype, device=g.device) if bias else None
    L = ampq.lib()
    need, ws = C.c_longlong(), None
    if sums:
        _check(L.ampq_norm_backward_workspace(device, rows, cols, C.byref(need)), "ampq_norm_backward_workspace")
        ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device=g.device)
    _check(L.ampq_norm_backward(device, stream, kind, _code(g), _code(weight) if weight is not None else _code(g), x.fmt if kept else ampq.FMT_BASE, g.data_ptr(), _pitch(g),
                                0 if kept else x.data_ptr(), 0 if kept else _pitch(x), *(_packed_args(x) if kept else (0, 0, 0, 0)), rows, cols,
                                _ptr(mean) if kind == ampq.NORM_LAYER else 0, rstd.data_ptr(), _ptr(weight), gx.data_ptr(), cols, _ptr(gw), _ptr(gb),
                                _ptr(ws), need.value), "ampq_norm_backward")
    return gx, gw if weight is not None else None, gb
