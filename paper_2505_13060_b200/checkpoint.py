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
import functools

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


def _device_of(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("tensors are on a CUDA device, got %s" % t.device)
    return t.device.index


_stream_of = torch._C._cuda_getCurrentRawStream  # the handle of torch's current stream on a device


def _code(t: torch.Tensor) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError("operands are float32 or bfloat16, got %s" % t.dtype)
    return code


def _pitch(t: torch.Tensor) -> int:
    """Elements between two rows of a matrix with contiguous rows."""
    rows, cols = t.shape
    return t.stride(0) if rows > 1 and cols > 0 else cols


def _matrix(t: torch.Tensor) -> torch.Tensor:
    """t as rows of its last dimension, without a copy where the layout allows it."""
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError("operands have at least one dimension")
        rows = 1
        for d in t.shape[:-1]:
            rows *= d
        t = t.reshape(rows, t.shape[-1])  # a view where it can be one
    if not t.is_contiguous():
        rows, cols = t.shape
        if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
            t = t.contiguous()
    return t


def _same_device(device: int, *others):
    for t in others:
        if t is not None and (not t.is_cuda or t.device.index != device):
            raise ValueError("operands are on one device, got cuda:%d and %s" % (device, t.device))


def _new_packed(rows: int, cols: int, fmt: int, device) -> Packed:
    groups = -(-cols // ampq.CKPT_GROUP)
    p = object.__new__(Packed)
    width = groups * ampq.CKPT_GROUP
    p.codes = torch.empty_strided((rows, width), (max(width, 1), 1), dtype=torch.uint8, device=device)   # half the time of torch.empty
    p.scales = torch.empty_strided((rows, groups), (max(groups, 1), 1), dtype=torch.uint8, device=device)
    p.cols, p.fmt = cols, fmt
    return p


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
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t):
    return 0 if t is None else t.data_ptr()


# The workspaces depend on sizes, types and alignment alone.
@functools.lru_cache(maxsize=4096)
def _weight_grad_bytes(device: int, code: int, misalignment: int, pitch: int, samples: int, rows: int, cols: int, outs: int) -> int:
    need = C.c_longlong()
    _check(ampq.lib().ampq_ckpt_weight_grad_workspace(device, code, misalignment, pitch, samples, rows, cols, outs, C.byref(need)),
           "ampq_ckpt_weight_grad_workspace")
    return need.value


@functools.lru_cache(maxsize=4096)
def _norm_backward_bytes(device: int, rows: int, cols: int) -> int:
    need = C.c_longlong()
    _check(ampq.lib().ampq_norm_backward_workspace(device, rows, cols, C.byref(need)), "ampq_norm_backward_workspace")
    return need.value


def pack(x: torch.Tensor, fmt: int = ampq.FMT_E4M3) -> Packed:
    """The 8-bit checkpoint of x."""
    m = _matrix(x)
    device = _device_of(m)
    rows, cols = m.shape
    p = _new_packed(rows, cols, fmt, m.device)
    _check(ampq.lib().ampq_ckpt_pack(device, _stream_of(device), _code(m), fmt, m.data_ptr(), rows, cols, _pitch(m), *_packed_args(p)),
           "ampq_ckpt_pack")
    return p


def unpack(p: Packed, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values a checkpoint stands for, [rows, cols]; exact in either type."""
    rows, cols = p.codes.shape[0], p.cols
    device = _device_of(p.codes)
    out = torch.empty(rows, cols, dtype=dtype, device=p.codes.device)
    _check(ampq.lib().ampq_ckpt_unpack(device, _stream_of(device), _code(out), p.fmt, *_packed_args(p), rows, cols, out.data_ptr(), cols),
           "ampq_ckpt_unpack")
    return out


def weight_grad(p: Packed, gy: torch.Tensor, samples: int = 1, bias: bool = False):
    """Weight gradients of a linear layer from the checkpoint of its input and the
    gradient of its output, one per sample: the rows are ``samples`` equal runs.
    Returns (gw [samples, outs, cols], gb [samples, outs] or None) in gy's type."""
    g = _matrix(gy)
    device = _device_of(g)
    _same_device(device, p.codes)
    total, outs = g.shape
    if samples < 1 or total != p.codes.shape[0] or total % samples:
        raise ValueError("%d gradient rows, %d checkpoint rows, %d samples" % (total, p.rows, samples))
    rows, cols, code, pitch, where, ptr = total // samples, p.cols, _code(g), _pitch(g), g.device, g.data_ptr()
    gw = torch.empty(samples, outs, cols, dtype=g.dtype, device=where)
    gb = torch.empty(samples, outs, dtype=g.dtype, device=where) if bias else None
    need = _weight_grad_bytes(device, code, ptr % 16, pitch, samples, rows, cols, outs)
    ws = torch.empty(need, dtype=torch.uint8, device=where) if need else None
    _check(ampq.lib().ampq_ckpt_weight_grad(device, _stream_of(device), code, p.fmt, ptr, pitch, *_packed_args(p), samples, rows, cols, outs,
                                            gw.data_ptr(), _ptr(gb), _ptr(ws), need), "ampq_ckpt_weight_grad")
    return gw, gb


def norm_forward(x: torch.Tensor, weight, bias, eps: float, kind: int = ampq.NORM_LAYER, fmt: int = ampq.FMT_BASE):
    """Layer norm or RMS norm over the last dimension.  Returns (y, mean, rstd, p):
    mean is None for an RMS norm, p the checkpoint of x or None for ``FMT_BASE``."""
    m = _matrix(x)
    device = _device_of(m)
    _same_device(device, weight, bias)
    where, code = m.device, _code(m)
    rows, cols = m.shape
    weight = _param(weight, cols)
    bias = _param(bias, cols, weight)
    y = torch.empty(x.shape, dtype=x.dtype, device=where)
    rstd = torch.empty(rows, dtype=torch.float32, device=where)
    mean = torch.empty(rows, dtype=torch.float32, device=where) if kind == ampq.NORM_LAYER else None
    p = _new_packed(rows, cols, fmt, where) if fmt != ampq.FMT_BASE else None
    pcode = _code(weight) if weight is not None else _code(bias) if bias is not None else code
    _check(ampq.lib().ampq_norm_forward(device, _stream_of(device), kind, code, pcode, fmt, m.data_ptr(), _pitch(m), rows, cols, _ptr(weight),
                                        _ptr(bias), eps, y.data_ptr(), cols, _ptr(mean), rstd.data_ptr(),
                                        *(_packed_args(p) if p is not None else (0, 0, 0, 0))), "ampq_norm_forward")
    return y, mean, rstd, p


def norm_backward(gy: torch.Tensor, x, mean, rstd: torch.Tensor, weight, kind: int = ampq.NORM_LAYER, bias: bool = True, bias_dtype=None):
    """Backward pass of ``norm_forward``; x is the input or its checkpoint.  Returns
    (gx, gw, gb): gw is None without a weight, gb unless a layer norm with a bias.
    They are in the weight's type; without a weight gb is in ``bias_dtype``, or gy's."""
    g = _matrix(gy)
    device = _device_of(g)
    rows, cols = g.shape
    kept = isinstance(x, Packed)
    if not kept:
        x = _matrix(x)
    _same_device(device, x.codes if kept else x, mean, rstd, weight)
    if (x.rows, x.cols) != (rows, cols) if kept else tuple(x.shape) != (rows, cols):
        raise ValueError("the input does not have the gradient's %d rows of %d columns" % (rows, cols))
    if not kept and x.dtype != g.dtype:
        raise TypeError("input and gradient are of one type, got %s and %s" % (x.dtype, g.dtype))
    layer = kind == ampq.NORM_LAYER
    for t in (rstd, mean) if layer else (rstd,):
        if t is None or t.dtype != torch.float32 or t.numel() != rows or not t.is_contiguous():
            raise ValueError("mean and rstd are as norm_forward returned them")
    where, code = g.device, _code(g)
    weight = _param(weight, cols)
    pdtype = weight.dtype if weight is not None else bias_dtype or g.dtype
    pcode = _CODE.get(pdtype)
    if pcode is None:
        raise TypeError("parameters are float32 or bfloat16, got %s" % pdtype)
    gx = torch.empty(gy.shape, dtype=g.dtype, device=where)
    bias = bias and layer
    gw = torch.empty(cols, dtype=pdtype, device=where) if weight is not None or bias else None
    gb = torch.empty(cols, dtype=pdtype, device=where) if bias else None
    need, ws = 0, None
    if gw is not None:
        need = _norm_backward_bytes(device, rows, cols)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=where)
    _check(ampq.lib().ampq_norm_backward(device, _stream_of(device), kind, code, pcode, x.fmt if kept else ampq.FMT_BASE, g.data_ptr(), _pitch(g),
                                         0 if kept else x.data_ptr(), 0 if kept else _pitch(x), *(_packed_args(x) if kept else (0, 0, 0, 0)),
                                         rows, cols, _ptr(mean) if layer else 0, rstd.data_ptr(), _ptr(weight), gx.data_ptr(), cols, _ptr(gw),
                                         _ptr(gb), _ptr(ws), need), "ampq_norm_backward")
    return gx, gw if weight is not None else None, gb


# -- differentiable forms ---------------------------------------------------------------------------------------------


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, fmt):
        y = torch.nn.functional.linear(x, weight, bias)
        p = pack(x.detach(), fmt) if weight.requires_grad else None
        ctx.save_for_backward(weight, *((p.codes, p.scales) if p is not None else ()))
        ctx.x_shape, ctx.fmt, ctx.bias = x.shape, fmt, bias is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        weight, *kept = ctx.saved_tensors
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        gx = gw = gb = None
        if need_x:
            gx = torch.matmul(gy, weight)
        if need_w:
            gw, gb = weight_grad(Packed(*kept, ctx.x_shape[-1], ctx.fmt), gy, bias=ctx.bias and need_b)
            gw = gw[0]
            gb = gb[0] if gb is not None else None
        elif need_b:
            gb = gy.reshape(-1, gy.shape[-1]).sum(0)
        return gx, gw, gb, None


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, kind, fmt):
        y, mean, rstd, p = norm_forward(x.detach(), weight, bias, eps, kind, fmt)
        ctx.kept = p is not None
        ctx.save_for_backward(weight, mean, rstd, *((p.codes, p.scales) if p is not None else (x,)))
        ctx.cols, ctx.kind, ctx.fmt = x.shape[-1], kind, fmt
        ctx.bias_dtype = bias.dtype if bias is not None else None
        ctx.shapes = [t.shape if t is not None else None for t in (weight, bias)]
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        weight, mean, rstd, *kept = ctx.saved_tensors
        need_b = ctx.needs_input_grad[2]
        x = Packed(*kept, ctx.cols, ctx.fmt) if ctx.kept else kept[0]
        gx, gw, gb = norm_backward(gy, x, mean, rstd, weight, ctx.kind, bias=need_b, bias_dtype=ctx.bias_dtype)
        gw, gb = (g.view(s) if g is not None else None for g, s in zip((gw, gb), ctx.shapes))   # [1, C] parameters too
        return gx, gw, gb, None, None, None


def autocast(*tensors):
    """Operands of a product as autocast would give them to torch's own: in its type, where it is on."""
    if not torch.is_autocast_enabled("cuda"):
        return tensors
    dtype = torch.get_autocast_dtype("cuda")
    return tuple(t.to(dtype) if t is not None and t.is_cuda and t.is_floating_point() and t.dtype != torch.float64 else t for t in tensors)


def linear(x: torch.Tensor, weight: torch.Tensor, bias=None, fmt: int = ampq.FMT_E4M3) -> torch.Tensor:
    """``torch.nn.functional.linear`` that keeps x for the backward pass in 8 bits:
    the weight's gradient is that of the decoded x, everything else is exact.  Under
    autocast the operands are cast first, as torch does."""
    x, weight, bias = autocast(x, weight, bias)
    if not torch.is_grad_enabled():
        return torch.nn.functional.linear(x, weight, bias)
    return _Linear.apply(x, weight, bias, fmt)


def layer_norm(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-5, fmt: int = ampq.FMT_E4M3) -> torch.Tensor:
    """Layer norm over the last dimension; x is kept for the backward pass in 8 bits,
    or in full with ``FMT_BASE``."""
    return _Norm.apply(x, weight, bias, eps, ampq.NORM_LAYER, fmt if torch.is_grad_enabled() else ampq.FMT_BASE)


def rms_norm(x: torch.Tensor, weight=None, eps: float = 1e-5, fmt: int = ampq.FMT_E4M3) -> torch.Tensor:
    """RMS norm over the last dimension; x is kept as in ``layer_norm``."""
    return _Norm.apply(x, weight, None, eps, ampq.NORM_RMS, fmt if torch.is_grad_enabled() else ampq.FMT_BASE)
