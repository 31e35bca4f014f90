"""The operators of a decoder's pass around its linear layers and norms, on torch tensors.

A calibration runs a model forward and backward; besides the linear layers and the
norms of whole rows (``checkpoint``) that takes the embedding in front, the norms of
queries and keys for each head with the position rotation, and a loss.  The loss here
needs no labels: the divergence from a teacher of which the top logits of each token
are known.  ``embedding``, ``head_norm`` and ``distill_loss`` are differentiable; the
other functions are the forward and backward passes on their own.

The calls of ``include/ampq.h`` (``ampq_embed_*``, ``ampq_head_norm_*``,
``ampq_distill_*``): operands are float32 or bfloat16, indices int32 or int64,
outputs and workspaces come from torch's caching allocator, and everything runs on
torch's current stream of the tensors' device.  No index is checked on the host (that
would wait for the device); the kernels use none that is out of range.  Everything can
be captured into a graph; a captured backward pass has leaves of its own, as any of
torch's.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct

import torch

from . import binding as ampq
from .checkpoint import Packed, _check, _code, _device_of, _matrix, _new_packed, _packed_args, _pitch, _ptr, _same_device, _stream_of

_INDEX = {torch.int32: ampq.I32, torch.int64: ampq.I64}


def _index_code(t: torch.Tensor) -> int:
    code = _INDEX.get(t.dtype)
    if code is None:
        raise TypeError("indices are int32 or int64, got %s" % t.dtype)
    return code


def _like(t: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor of t's shape and type.  (Like a tensor or with strides torch makes one in half the time.)"""
    return torch.empty_like(t) if t.is_contiguous() else _new(t.shape, t.dtype, t.device)


def _new(shape, dtype, where) -> torch.Tensor:
    strides, n = [], 1
    for d in reversed(shape):
        strides.append(n)
        n *= d or 1
    return torch.empty_strided(shape, strides[::-1], dtype=dtype, device=where)


# -- embedding --------------------------------------------------------------------------------------------------------


def embed(tokens: torch.Tensor, weight: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """``weight[tokens] * scale`` [*tokens.shape, columns], rounded once.  A token outside the table has a row of NaN."""
    if weight.dim() != 2:
        raise ValueError("a table has rows and columns, got %s" % (tuple(weight.shape),))
    w = _matrix(weight)
    device = _device_of(w)
    _same_device(device, tokens)
    index, code = _index_code(tokens), _code(w)
    t = tokens if tokens.is_contiguous() else tokens.contiguous()
    vocab, cols = w.shape
    y = _new((*tokens.shape, cols), w.dtype, w.device)
    _check(ampq.lib().ampq_embed_forward(device, _stream_of(device), code, index, t.data_ptr(), t.numel(), w.data_ptr(), _pitch(w), vocab, cols, scale,
                                         y.data_ptr(), cols), "ampq_embed_forward")
    return y


@functools.lru_cache(maxsize=4096)
def _embed_backward_bytes(device: int, code: int, n: int, vocab: int, cols: int) -> int:
    need = C.c_longlong()
    _check(ampq.lib().ampq_embed_backward_workspace(device, code, n, vocab, cols, C.byref(need)), "ampq_embed_backward_workspace")
    return need.value


def embed_backward(tokens: torch.Tensor, gy: torch.Tensor, vocab: int, scale: float = 1.0, padding_idx=None) -> torch.Tensor:
    """The table's gradient [vocab, columns] from that of ``embed``'s output, the same bits every time.  The row of
    ``padding_idx`` is zero, as are those of no token."""
    if tuple(gy.shape[:-1]) != tuple(tokens.shape) or gy.dim() < 1:
        raise ValueError("a gradient row for each token: tokens %s, gradient %s" % (tuple(tokens.shape), tuple(gy.shape)))
    padding = -1 if padding_idx is None else padding_idx
    if padding_idx is not None and not 0 <= padding_idx < vocab:
        raise ValueError("padding_idx %d is no row of a table of %d" % (padding_idx, vocab))
    g = _matrix(gy)
    device = _device_of(g)
    _same_device(device, tokens)
    index, code = _index_code(tokens), _code(g)
    t = tokens if tokens.is_contiguous() else tokens.contiguous()
    n, cols = g.shape
    gw = _new((vocab, cols), g.dtype, g.device)
    need = _embed_backward_bytes(device, code, n, vocab, cols)
    ws = _new((need,), torch.uint8, g.device)
    _check(ampq.lib().ampq_embed_backward(device, _stream_of(device), code, index, t.data_ptr(), n, g.data_ptr(), _pitch(g), vocab, cols, scale, padding,
                                          gw.data_ptr(), ws.data_ptr(), need), "ampq_embed_backward")
    return gw


# -- norms of queries and keys, with the position rotation ---------------------------------------------------------------


def rotary_table(length: int, rot: int, base: float = 10000.0, device="cuda"):
    """(cos, sin) [length, rot / 2] in fp32 of the angles position * base^(-2 i / rot), computed in 64 bits."""
    if rot < 0 or rot % 2 or length < 0:
        raise ValueError("%d positions of %d columns: columns are turned in pairs" % (length, rot))
    freq = float(base) ** (-torch.arange(rot // 2, device=device, dtype=torch.float64) * 2 / max(rot, 1))
    angle = torch.arange(length, device=device, dtype=torch.float64)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _by_token(x: torch.Tensor):
    """x [..., tokens, heads, columns] as [batch, tokens, heads, columns], in place where the layout allows it."""
    if x.dim() != 4:
        if x.dim() < 3:
            raise ValueError("queries and keys are [..., tokens, heads, columns], got %s" % (tuple(x.shape),))
        batch = 1
        for d in x.shape[:-3]:
            batch *= d
        x = x.reshape(batch, *x.shape[-3:])
    if x.stride(3) != 1 and x.shape[3] > 1:
        x = x.contiguous()
    return x


def _rotation(cos, sin, positions, batch: int, tokens: int, device: int, leading):
    """(pointer of cos, of sin, columns turned, table rows, pointer of the positions, their index type, elements between
    batches), and the tensors that these are of."""
    if cos is None and sin is None:
        return (0, 0, 0, 0, 0, ampq.I64, 0), ()
    if cos is None or sin is None or cos.dim() != 2 or cos.shape != sin.shape:
        raise ValueError("cos and sin are tables [positions, pairs] of one shape")
    if cos.dtype != torch.float32 or sin.dtype != torch.float32:
        raise TypeError("cos and sin are float32, got %s and %s" % (cos.dtype, sin.dtype))
    _same_device(device, cos, sin, positions)
    if not cos.is_contiguous() or cos.data_ptr() % 16:
        cos = cos.clone(memory_format=torch.contiguous_format)
    if not sin.is_contiguous() or sin.data_ptr() % 16:
        sin = sin.clone(memory_format=torch.contiguous_format)
    angles, pairs = cos.shape
    if positions is None:
        return (cos.data_ptr(), sin.data_ptr(), 2 * pairs, angles, 0, ampq.I64, 0), (cos, sin)
    index, shape = _index_code(positions), positions.shape
    if len(shape) == 1 and shape[0] == tokens:
        stride = 0
    elif shape[-1:] == (tokens,) and len(shape) <= len(leading) + 1 and all(a in (1, b) for a, b in zip(reversed(shape[:-1]), reversed(leading))):
        if shape != (*leading, tokens):
            positions = positions.expand(*leading, tokens)
        positions = positions if len(leading) == 1 else positions.reshape(batch, tokens)
        stride = positions.stride(0) if batch > 1 else 0
    else:
        raise ValueError("positions are [%d] or as many as %s, got %s" % (tokens, (*leading, tokens), tuple(shape)))
    if tokens > 1 and positions.stride(-1) != 1:
        positions = positions.contiguous()
        stride = tokens if positions.dim() == 2 else 0
    return (cos.data_ptr(), sin.data_ptr(), 2 * pairs, angles, positions.data_ptr(), index, stride), (cos, sin, positions)


def _head_weight(w, cols: int, like):
    if w is None:
        return None
    if w.numel() != cols:
        raise ValueError("a norm over heads of %d columns has a weight of that many elements, got %s" % (cols, tuple(w.shape)))
    if like is not None and like.dtype != w.dtype:
        raise TypeError("weights are of one type, got %s and %s" % (like.dtype, w.dtype))
    return w if w.is_contiguous() else w.contiguous()


def _strides(t):
    """Pointer of t [batch, tokens, heads, columns] and its strides; those of single elements have no meaning."""
    if t is None:
        return 0, 0, 0, 0
    (b, n, h, _), (sb, sn, sh, _) = t.shape, t.stride()
    return t.data_ptr(), sb if b > 1 else 0, sn if n > 1 else 0, sh if h > 1 else 0


_HEADS = struct.Struct("%dq" % (C.sizeof(ampq.Heads) // 8))   # its fields in order, in a third of the time that the class takes


def _side(out, rstd, w, x=None, gy=None, gw=None, kept=None):
    """The bytes of an ``ampq_heads`` (``binding.Heads``)."""
    ptr, *strides = _strides(out)
    return _HEADS.pack(out.shape[2], *_strides(x), *_strides(gy), ptr, *strides, _ptr(w), _ptr(gw), rstd.data_ptr(),
                       *(_packed_args(kept) if kept is not None else (0, 0, 0, 0)))


def head_norm_forward(q: torch.Tensor, k, wq=None, wk=None, cos=None, sin=None, positions=None, eps: float = 1e-5, interleaved: bool = False,
                      fmt: int = ampq.FMT_BASE):
    """RMS norm of each head of q [..., tokens, heads, columns] and of k [..., tokens, key heads, columns] (or None), with the
    weights wq and wk [columns] that their heads share (None for ones), and the rotation of the first ``2 * cos.shape[1]``
    columns by the angles of the tokens' positions: row ``positions[..., t]`` of the tables cos and sin
    (``rotary_table``), row t without positions, no rotation without tables.  Positions are [tokens] or [..., tokens],
    where dimensions of 1 hold for all of a batch.  Pairs are (i, i + half) or, ``interleaved``, (2 i, 2 i + 1).

    Returns (yq, yk, rq, rk, pq, pk): the outputs, the reciprocals [..., tokens, heads] of the root mean squares, and the
    checkpoints of q and k (a row for each head) or None for ``FMT_BASE``."""
    x = _by_token(q)
    device = _device_of(x)
    batch, tokens, heads, cols = x.shape
    code, where = _code(x), x.device
    _same_device(device, k, wq, wk)
    if k is not None:
        if q.shape[:-2] != k.shape[:-2] or k.shape[-1] != cols:
            raise ValueError("queries %s and keys %s differ in more than their heads" % (tuple(q.shape), tuple(k.shape)))
        if k.dtype != q.dtype:
            raise TypeError("queries and keys are of one type, got %s and %s" % (q.dtype, k.dtype))
    wq = _head_weight(wq, cols, None)
    wk = _head_weight(wk, cols, wq) if k is not None else None
    turn, held = _rotation(cos, sin, positions, batch, tokens, device, q.shape[:-3])
    pcode = _code(wq) if wq is not None else _code(wk) if wk is not None else code

    def side(x, w):
        y = _like(x)
        r = _new(x.shape[:3], torch.float32, where)
        p = _new_packed(r.numel(), cols, fmt, where) if fmt != ampq.FMT_BASE else None
        return y, r, p, _side(y, r, w, x=x, kept=p)

    yq, rq, pq, first = side(x, wq)
    yk = rk = pk = second = None
    if k is not None:
        k4 = _by_token(k)
        yk, rk, pk, second = side(k4, wk)
    _check(ampq.lib().ampq_head_norm_forward(device, _stream_of(device), code, pcode, turn[5], fmt, 1 if interleaved else 0, batch, tokens, cols, turn[2], turn[0],
                                             turn[1], turn[3], turn[4], turn[6], eps, first, second), "ampq_head_norm_forward")
    if q.dim() != 4:
        yq, rq = yq.view(q.shape), rq.view(q.shape[:-1])
        if k is not None:
            yk, rk = yk.view(k.shape), rk.view(k.shape[:-1])
    return yq, yk, rq, rk, pq, pk


@functools.lru_cache(maxsize=4096)
def _head_norm_backward_bytes(device: int, batch: int, tokens: int, cols: int) -> int:
    need = C.c_longlong()
    _check(ampq.lib().ampq_head_norm_backward_workspace(device, batch, tokens, cols, C.byref(need)), "ampq_head_norm_backward_workspace")
    return need.value


def head_norm_backward(gq: torch.Tensor, gk, q, k, rq: torch.Tensor, rk=None, wq=None, wk=None, cos=None, sin=None, positions=None, interleaved: bool = False,
                       weight_grads: bool = True):
    """Backward pass of ``head_norm_forward``; q and k are the inputs or their checkpoints, gq and gk the gradients of the
    outputs.  Returns (gxq, gxk, gwq, gwk), the last two in their weight's type, None without one (or without ``weight_grads``)."""
    g = [_by_token(gq), _by_token(gk) if gk is not None else None]
    device = _device_of(g[0])
    batch, tokens, _, cols = g[0].shape
    code = _code(g[0])
    if gk is not None and (gq.shape[:-2] != gk.shape[:-2] or gk.shape[-1] != cols or gk.dtype != gq.dtype):
        raise ValueError("the gradients of queries %s %s and keys %s %s differ in more than their heads" % (tuple(gq.shape), gq.dtype, tuple(gk.shape), gk.dtype))
    if (gk is None) != (k is None) or (gk is None) != (rk is None):
        raise ValueError("keys have a gradient, an input and rk, or none of them")
    kept = isinstance(q, Packed)
    if k is not None and (isinstance(k, Packed) != kept or (kept and k.fmt != q.fmt)):
        raise ValueError("queries and keys are kept alike")
    wq = _head_weight(wq, cols, None)
    wk = _head_weight(wk, cols, wq) if gk is not None else None
    _same_device(device, g[1], rq, rk, wq, wk, *((q.codes, k.codes if k is not None else None) if kept else (q, k)))
    turn, held = _rotation(cos, sin, positions, batch, tokens, device, gq.shape[:-3])
    pcode = _code(wq) if wq is not None else _code(wk) if wk is not None else code
    gx, gw, sides = [None, None], [None, None], [None, None]
    inputs = []
    for i, (t, x, r, w) in enumerate(zip(g, (q, k), (rq, rk), (wq, wk))):
        if t is None:
            continue
        rows = t.shape[0] * t.shape[1] * t.shape[2]
        if kept:
            if (x.rows, x.cols) != (rows, cols):
                raise ValueError("a checkpoint of %d rows of %d columns for %d of %d" % (x.rows, x.cols, rows, cols))
        else:
            x = _by_token(x)
            inputs.append(x)   # a copy lives until the call
            if x.shape != t.shape or x.dtype != t.dtype:
                raise ValueError("input %s %s and gradient %s %s" % (tuple(x.shape), x.dtype, tuple(t.shape), t.dtype))
        if r.dtype != torch.float32 or r.numel() != rows or not r.is_contiguous():
            raise ValueError("rq and rk are as head_norm_forward returned them")
        gx[i] = _like(t)
        gw[i] = _like(w) if w is not None and weight_grads else None
        sides[i] = _side(gx[i], r, w, x=None if kept else x, gy=t, gw=gw[i], kept=x if kept else None)
    need = _head_norm_backward_bytes(device, batch, tokens, cols) if gw[0] is not None or gw[1] is not None else 0
    ws = _new((need,), torch.uint8, g[0].device) if need else None
    _check(ampq.lib().ampq_head_norm_backward(device, _stream_of(device), code, pcode, turn[5], q.fmt if kept else ampq.FMT_BASE, 1 if interleaved else 0, batch,
                                              tokens, cols, turn[2], turn[0], turn[1], turn[3], turn[4], turn[6], *sides, _ptr(ws), need),
           "ampq_head_norm_backward")
    if gq.dim() != 4:
        gx[0] = gx[0].view(gq.shape)
        gx[1] = gx[1].view(gk.shape) if gk is not None else None
    return gx[0], gx[1], gw[0], gw[1]


# -- distillation -------------------------------------------------------------------------------------------------------


def _lists(logits, indices, teacher):
    """Matrices of the three operands, and where they are."""
    if logits.dim() < 1 or indices.dim() < 1 or indices.shape != teacher.shape or indices.shape[:-1] != logits.shape[:-1]:
        raise ValueError("a list of columns and of the teacher's logits for each row: logits %s, indices %s, teacher %s"
                         % (tuple(logits.shape), tuple(indices.shape), tuple(teacher.shape)))
    s, i, t = _matrix(logits), _matrix(indices), _matrix(teacher)
    device = _device_of(s)
    _same_device(device, i, t)
    return s, i, t, device, (_code(s), _code(t), _index_code(i))


def _list_args(s, i, t):
    rows, cols = s.shape
    return s.data_ptr(), _pitch(s), rows, cols, i.data_ptr(), _pitch(i), t.data_ptr(), _pitch(t), i.shape[1]


def list_length(logits: torch.Tensor, top: int) -> int:
    """Length of a list of the ``top`` largest of logits [..., classes]; raises where ``distill_forward`` would refuse the
    logits or the list."""
    if logits.dim() < 1:
        raise ValueError("logits are [..., classes], got %s" % (tuple(logits.shape),))
    _device_of(logits)
    _code(logits)
    top = min(top, logits.shape[-1])
    if top > ampq.DISTILL_MAX_TOP:
        raise ValueError("lists hold up to %d columns, got %d" % (ampq.DISTILL_MAX_TOP, top))
    return top


def distill_forward(logits: torch.Tensor, indices: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0):
    """Divergence of softmax(logits / T) [..., vocabulary] from a teacher's: the columns ``indices`` [..., k] (negative: no
    entry) with the teacher's logits ``teacher`` [..., k], whose probabilities are those of softmax(teacher / T) over the
    row's entries.  Returns (loss [...] in fp32, times T^2; stats [..., 2] for the backward pass)."""
    s, i, t, device, codes = _lists(logits, indices, teacher)
    leading = logits.shape[:-1]
    loss, stats = _new(leading, torch.float32, s.device), _new((*leading, 2), torch.float32, s.device)
    _check(ampq.lib().ampq_distill_forward(device, _stream_of(device), *codes, *_list_args(s, i, t), temperature, loss.data_ptr(), stats.data_ptr()),
           "ampq_distill_forward")
    return loss, stats


def distill_backward(gl: torch.Tensor, logits: torch.Tensor, indices: torch.Tensor, teacher: torch.Tensor, stats: torch.Tensor, temperature: float = 1.0):
    """Gradient of the logits from that of the losses, gl [...] (a number expanded to the rows is read in place).  Where a
    list names a column that is none, its other columns are NaN, and what is not listed has the first term alone."""
    s, i, t, device, codes = _lists(logits, indices, teacher)
    if gl.shape != logits.shape[:-1] or stats.shape != (*logits.shape[:-1], 2):
        raise ValueError("a gradient and statistics for each row: logits %s, gl %s, stats %s" % (tuple(logits.shape), tuple(gl.shape), tuple(stats.shape)))
    if gl.dtype != torch.float32 or stats.dtype != torch.float32:
        raise TypeError("losses and statistics are float32, got %s and %s" % (gl.dtype, stats.dtype))
    _same_device(device, gl, stats)
    rows = s.shape[0]
    if rows > 1 and all(d == 1 or st == 0 for d, st in zip(gl.shape, gl.stride())):
        stride = 0
    else:
        gl = gl if gl.is_contiguous() else gl.contiguous()
        stride = 1
    stats = stats if stats.is_contiguous() else stats.contiguous()
    gs = _like(logits)
    _check(ampq.lib().ampq_distill_backward(device, _stream_of(device), *codes, gl.data_ptr(), stride, *_list_args(s, i, t), stats.data_ptr(), temperature,
                                            gs.data_ptr(), s.shape[1]), "ampq_distill_backward")
    return gs


# -- differentiable forms -------------------------------------------------------------------------------------------------


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, padding_idx):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale, ctx.padding_idx = weight.shape[0], scale, padding_idx
        return embed(tokens, weight.detach(), scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        tokens, = ctx.saved_tensors
        return None, embed_backward(tokens, gy, ctx.vocab, ctx.scale, ctx.padding_idx), None, None


class _HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps, interleaved, fmt):
        yq, yk, rq, rk, pq, pk = head_norm_forward(q.detach(), k.detach() if k is not None else None, wq, wk, cos, sin, positions, eps, interleaved, fmt)
        kept = [(p.codes, p.scales) if p is not None else (x, None) for p, x in ((pq, q), (pk, k))]
        ctx.save_for_backward(wq, wk, cos, sin, positions, rq, rk, *kept[0], *kept[1])
        ctx.cols, ctx.fmt, ctx.interleaved = q.shape[-1], fmt, interleaved
        return yq, yk

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        wq, wk, cos, sin, positions, rq, rk, *kept = ctx.saved_tensors
        x = [Packed(a, b, ctx.cols, ctx.fmt) if b is not None else a for a, b in (kept[:2], kept[2:])]
        gxq, gxk, gwq, gwk = head_norm_backward(gq, gk, x[0], x[1], rq, rk, wq, wk, cos, sin, positions, ctx.interleaved, any(ctx.needs_input_grad[2:4]))
        return gxq, gxk, gwq, gwk, None, None, None, None, None, None


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, indices, teacher, temperature):
        loss, stats = distill_forward(logits.detach(), indices, teacher, temperature)
        ctx.save_for_backward(logits, indices, teacher, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gl):
        return distill_backward(gl, *ctx.saved_tensors, ctx.temperature), None, None, None


def embedding(tokens: torch.Tensor, weight: torch.Tensor, scale: float = 1.0, padding_idx=None) -> torch.Tensor:
    """``embed``, differentiable in the table: the gradient's rows are added in an order that the tokens fix.  The row
    ``padding_idx`` gets no gradient."""
    if padding_idx is not None and not 0 <= padding_idx < weight.shape[0]:
        raise ValueError("padding_idx %d is no row of a table of %d" % (padding_idx, weight.shape[0]))
    return _Embedding.apply(tokens, weight, scale, padding_idx)


def head_norm(q: torch.Tensor, k=None, wq=None, wk=None, cos=None, sin=None, positions=None, eps: float = 1e-5, interleaved: bool = False,
              fmt: int = ampq.FMT_E4M3):
    """The outputs (yq, yk) of ``head_norm_forward``, differentiable; q and k are kept for the backward pass in 8 bits, or
    in full with ``FMT_BASE``.  The default is that of ``checkpoint.linear`` and the norms there: the gradients are those of
    the decoded inputs.  (The module ``HeadNorm`` keeps them in full by default.)  cos and sin are constants."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (cos, sin)):
        raise ValueError("the angles are a constant here: detach them")
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, wq, wk))
    return _HeadNorm.apply(q, k, wq, wk, cos, sin, positions, eps, interleaved, fmt if keep else ampq.FMT_BASE)


def distill_loss(logits: torch.Tensor, indices: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0) -> torch.Tensor:
    """The losses [...] of ``distill_forward``, differentiable in the logits.  The teacher is a constant."""
    if torch.is_grad_enabled() and teacher.requires_grad:
        raise ValueError("the teacher's logits are a constant here: detach them")
    return _DistillLoss.apply(logits, indices, teacher, temperature)


# -- modules --------------------------------------------------------------------------------------------------------------


class ScaledEmbedding(torch.nn.Embedding):
    """``torch.nn.Embedding`` whose rows are multiplied by ``scale`` and whose gradient is the same bits every time."""

    def __init__(self, num_embeddings: int, embedding_dim: int, scale: float = 1.0, padding_idx=None, **kwargs):
        super().__init__(num_embeddings, embedding_dim, padding_idx=padding_idx, **kwargs)
        if self.max_norm is not None or self.scale_grad_by_freq or self.sparse:
            raise ValueError("max_norm, scale_grad_by_freq and sparse are not for this module")
        self.scale = scale

    def forward(self, input):
        return embedding(input, self.weight, self.scale, self.padding_idx)


class HeadNorm(torch.nn.Module):
    """Norms of queries and keys for each head with the position rotation, between the layers that make them and their
    product.  Its inputs are kept in full for the backward pass unless ``fmt`` names a format, unlike ``head_norm``'s, which
    are kept in E4M3 by default; in a calibration with checkpoints (``hooks.Calibrator``) they are in its format."""

    def __init__(self, cols: int, eps: float = 1e-5, interleaved: bool = False, device=None, dtype=None):
        super().__init__()
        self.weight_q = torch.nn.Parameter(torch.ones(cols, device=device, dtype=dtype))
        self.weight_k = torch.nn.Parameter(torch.ones(cols, device=device, dtype=dtype))
        self.eps, self.interleaved = eps, interleaved

    def forward(self, q, k, cos=None, sin=None, positions=None, fmt: int = ampq.FMT_BASE):
        return head_norm(q, k, self.weight_q, self.weight_k, cos, sin, positions, self.eps, self.interleaved, fmt)
