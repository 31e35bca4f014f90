"""Calibration of a PyTorch model through module hooks (Algorithm 1 step 2:
"wrap the model", then one high-precision forward and backward per sample).

``Calibrator`` registers every ``torch.nn.Linear`` of a model as a linear layer
of a scoring context and every ``BatchedMatmul`` (a module that only wraps
``torch.matmul``, so that the attention products Q K^T and P V are visible to
hooks) as a batched GEMM with operands X0, X1 (Sec. 2.2).  While a sample runs, a forward hook keeps the layer input X
and a backward hook receives dL/dX and dL/dY; the sample's weight gradient
dL/dW = dL/dY^T X is formed by a torch matmul (the GEMM that produces a gradient
is not part of the scoring path) and both operands of the layer are streamed to
``ampq_stream_sample``, so the R per-sample weight gradients never exist at the
same time: a sample's tensors are released as soon as the library's work on
them is ordered before any reuse of their memory -- at once when the context
runs on torch's current stream (the caching allocator hands a freed block only
to later work of the same stream), else when a CUDA event recorded on the
context's stream after the sample has completed, with at most two samples
pending.  Everything the method computes happens in the CUDA library; this
module only moves pointers.

With ``checkpoint=FMT_E4M3`` (or ``FMT_E5M2``) the calibration keeps the inputs of
the linear layers and of ``torch.nn.LayerNorm`` and ``torch.nn.RMSNorm`` modules
(those with a forward of their own apart, which run as without checkpoints) in
8 bits between the forward and the backward pass -- the memory that calibration
needs beyond the model (Sec. 1) -- and forms the sample's weight gradients and the
norms' gradients from there (``checkpoint``).  Each layer keeps its own 33/32 byte per
element: half of bf16 for an input with one reader, more than one shared bf16 tensor
for an input that three layers read (q, k and v).  A sample's peak, 24 linear layers
of 2048 in a row: 16.4 inputs of a layer against 27 without checkpoints; four
7B-shaped blocks, whose attention and activation keep theirs in full: 1339 MB against
1373.

What is scored is what the backward pass has: the decoded inputs.  An element in the
normal range of its group's scale is off by at most half a step of the format (2^-4 of
itself in E4M3, 2^-3 in E5M2), so where dL/dX is exact and such elements carry the
sum, the model's term S of an input operand is off by at most 13 % (27 %).  Smaller
elements may lose more of themselves, a weight's S goes by dL/dW, whose sums can
cancel, and behind a norm dL/dX itself follows the decoded input: no such bound
exists there.  Measured on the four blocks against a calibration without checkpoints:
S of inputs and of weights off by 0.1 % on average, 0.2 % at worst in E4M3, 0.4 % and
0.6 % in E5M2.  The measured term of a
tensor that was already rounded says nothing, so the pass scores the model's term
alone (``set_measured(False)``; the context's next pass has its own setting again).

``quantised(...)`` runs the model with chosen layers' inputs and weights replaced
by their FP8-rounded values (``ampq_fake_quant``), which is how the predicted
loss MSE is checked against a measured one (Sec. 3.2).
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as ampq
from . import checkpoint as ckpt


class BatchedMatmul(torch.nn.Module):
    """``torch.matmul(a, b)`` as a module: a batched GEMM layer Y = X0 (x) X1 whose
    two operands and their gradients the calibrator can see."""

    def forward(self, a, b):
        return torch.matmul(a, b)


class _ScoredLinear(torch.autograd.Function):
    """A linear layer of a calibration with 8-bit checkpoints: its input is kept
    packed, its backward pass streams the layer's two operands."""

    @staticmethod
    def forward(ctx, x, weight, bias, calibrator, idx):
        y = torch.nn.functional.linear(x, weight, bias)
        p = ckpt.pack(x.detach(), calibrator.checkpoint)   # refuses what cannot be kept: a layer is not left out silently
        ctx.save_for_backward(weight, p.codes, p.scales)
        ctx.x_shape, ctx.calibrator, ctx.idx, ctx.r = x.shape, calibrator, idx, calibrator._r
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        weight, codes, scales = ctx.saved_tensors
        cal, (need_x, need_w, need_b) = ctx.calibrator, ctx.needs_input_grad[:3]
        p = ckpt.Packed(codes, scales, ctx.x_shape[-1], cal.checkpoint)
        gx = torch.matmul(gy, weight)
        gw, gb = ckpt.weight_grad(p, gy, bias=need_b)
        if cal._r is not None:
            if ctx.idx in cal._done:
                raise RuntimeError("layer %s was used twice in sample %d: it has one pair of operands" % (cal.modules[ctx.idx][0], ctx.r))
            cal._done.add(ctx.idx)
            cal._stream_linear(ctx.idx, ctx.r, ckpt.unpack(p, weight.dtype), gx, weight.detach(), gw[0])
        return gx if need_x else None, gw[0] if need_w else None, gb[0] if need_b else None, None, None


class Calibrator:
    def __init__(self, ctx: "ampq.Context", model: torch.nn.Module, R: int, checkpoint: int = ampq.FMT_BASE):
        if checkpoint not in (ampq.FMT_BASE, ampq.FMT_E4M3, ampq.FMT_E5M2):
            raise ValueError("checkpoint is FMT_BASE (inputs kept in full), FMT_E4M3 or FMT_E5M2")
        self.ctx, self.model, self.R, self.checkpoint = ctx, model, R, checkpoint
        self._replaced = []   # (module, the forward that keeps its input in 8 bits), in place while a sample runs
        self.modules, self.layer_ids = [], []
        for name, m in model.named_modules():
            if isinstance(m, torch.nn.Linear):
                self.modules.append((name, m))
                self.layer_ids.append(ctx.register_layer(ampq.LINEAR, name, R))
            elif isinstance(m, BatchedMatmul):
                self.modules.append((name, m))
                self.layer_ids.append(ctx.register_layer(ampq.BGEMM, name, R))
        self._r = None
        self._x = {}
        self._done = set()   # layers with a checkpoint that were streamed in the current sample
        self._keep = []      # tensors the library borrowed during the current sample
        self._pending = []   # (event on the context's stream, tensors) of earlier samples
        self._handles = []

    # -- lifetime of borrowed tensors -------------------------------------------
    def _same_stream(self) -> bool:
        return torch.cuda.current_stream().cuda_stream == self.ctx.stream

    def _borrowed(self, *tensors):
        """Holds what the library's work on the context's stream reads until the sample is over; on torch's own stream
        that work comes before any reuse of the memory, and nothing is held."""
        if not self._same_stream():
            self._keep += tensors

    def _release_sample(self):
        """Called when a sample's block ends: nothing more will be launched on its tensors."""
        if not self._keep:
            return
        if self._same_stream():
            self._keep = []   # stream order protects the memory
            return
        ev = torch.cuda.Event()
        ev.record(torch.cuda.ExternalStream(self.ctx.stream))
        self._pending.append((ev, self._keep))
        self._keep = []
        self._pending = [(e, t) for e, t in self._pending if not e.query()]
        while len(self._pending) > 2:
            self._pending.pop(0)[0].synchronize()

    # -- hooks ----------------------------------------------------------------
    def _fwd(self, idx):
        def hook(module, inputs, output):
            if self._r is not None:
                self._x[idx] = tuple(t.detach() for t in inputs) if isinstance(module, BatchedMatmul) else inputs[0].detach()
        return hook

    def _bwd(self, idx):
        def hook(module, grad_input, grad_output):
            if self._r is None:
                return
            if not self._same_stream():   # the library's stream reads what torch's stream has just produced
                torch.cuda.ExternalStream(self.ctx.stream).wait_stream(torch.cuda.current_stream())
            if isinstance(module, BatchedMatmul):   # both operands belong to the sample
                lid = self.layer_ids[idx]
                for k, (x, gx) in enumerate(zip(self._x.pop(idx), grad_input)):
                    x = x.contiguous()
                    gx = (torch.zeros_like(x) if gx is None else gx.detach().reshape(x.shape)).contiguous()
                    self.ctx.stream_sample(lid, k, self._r, ampq.torch_dtype_code(x), x.data_ptr(), gx.data_ptr(), x.numel())
                    self._borrowed(x, gx)
                return
            x = self._x.pop(idx)
            gy = grad_output[0].detach()
            gx = grad_input[0]
            w = module.weight.detach()
            if gx is None:   # the model input needs no gradient: form dL/dX here
                gx = gy.reshape(-1, gy.shape[-1]) @ w
            gw = gy.reshape(-1, gy.shape[-1]).t() @ x.reshape(-1, x.shape[-1])
            self._stream_linear(idx, self._r, x, gx.detach(), w, gw)
        return hook

    def _stream_linear(self, idx, r, x, gx, w, gw):
        """Streams both operands of a linear layer for sample r."""
        if not self._same_stream():
            torch.cuda.ExternalStream(self.ctx.stream).wait_stream(torch.cuda.current_stream())
        x, w, gw = x.contiguous(), w.contiguous(), gw.contiguous()
        gx = gx.reshape(x.shape).contiguous()
        code = ampq.torch_dtype_code(x)
        lid = self.layer_ids[idx]
        self.ctx.stream_sample(lid, 0, r, code, x.data_ptr(), gx.data_ptr(), x.numel())
        self.ctx.stream_sample(lid, 1, r, code, w.data_ptr(), gw.data_ptr(), w.numel())
        self._borrowed(x, gx, w, gw)

    # -- 8-bit checkpoints ------------------------------------------------------
    @staticmethod
    def _plain(module, base) -> bool:
        """Whether a module computes what its base class does: subclasses with a forward of their own and modules that
        somebody has wrapped already run as they are."""
        return isinstance(module, base) and type(module).forward is base.forward and "forward" not in module.__dict__

    def _find_replaced(self):
        """The linear layers and norms that go through the calls that keep their input in 8 bits."""
        fmt = self.checkpoint
        self._replaced = []

        def scored():
            return self._r is not None and torch.is_grad_enabled()

        types = (torch.float32, torch.bfloat16)

        def known(x, m):   # a norm that the library has; torch runs the others, or says what is wrong with them
            params = [t for t in (m.weight, getattr(m, "bias", None)) if t is not None]
            return (scored() and not torch.is_autocast_enabled("cuda") and x.is_cuda and x.dtype in types and x.shape[-1:] == m.normalized_shape
                    and all(t.device == x.device and t.dtype in types and t.dtype == params[0].dtype for t in params))

        for idx, (_, m) in enumerate(self.modules):
            if self._plain(m, torch.nn.Linear):

                def linear(input, m=m, idx=idx, plain=m.forward):   # the module's own name for its argument
                    return _ScoredLinear.apply(*ckpt.autocast(input, m.weight, m.bias), self, idx) if scored() else plain(input)

                self._replaced.append((m, linear))
        for m in self.model.modules():
            if (self._plain(m, torch.nn.LayerNorm) or self._plain(m, torch.nn.RMSNorm)) and len(m.normalized_shape) == 1 and m.normalized_shape[0] <= ampq.NORM_MAX_COLS:

                def layer_norm(input, m=m, plain=m.forward):
                    return ckpt.layer_norm(input, m.weight, m.bias, m.eps, fmt) if known(input, m) else plain(input)

                def rms_norm(x, m=m, plain=m.forward):
                    # without an eps of its own the module takes that of fp32, in which it computes, whatever x's type
                    return ckpt.rms_norm(x, m.weight, torch.finfo(torch.float32).eps if m.eps is None else m.eps, fmt) if known(x, m) else plain(x)

                self._replaced.append((m, layer_norm if isinstance(m, torch.nn.LayerNorm) else rms_norm))

    def _remove_hooks(self):
        for h in self._handles:
            h.remove()
        self._handles = []

    def begin(self):
        self._remove_hooks()   # of a pass that was never ended
        if self.checkpoint != ampq.FMT_BASE:
            self._find_replaced()
        replaced = {m for m, _ in self._replaced}
        for idx, (_, m) in enumerate(self.modules):
            if m in replaced:
                continue
            self._handles.append(m.register_forward_hook(self._fwd(idx)))
            self._handles.append(m.register_full_backward_hook(self._bwd(idx)))
        self.ctx.stream_begin(measured=None if self.checkpoint == ampq.FMT_BASE else False)

    @contextlib.contextmanager
    def sample(self, r: int):
        """Run one sample's forward and backward inside this block."""
        for m, _ in self._replaced:
            if "forward" in m.__dict__:
                raise RuntimeError("a module's forward was replaced after begin()")
        self._r = r
        try:
            for m, forward in self._replaced:
                m.forward = forward
            yield
        finally:
            for m, _ in self._replaced:
                m.__dict__.pop("forward", None)   # the class's again
            self._r = None
            self._x.clear()
            self._done.clear()
            self._release_sample()

    def end(self):
        self._remove_hooks()
        self._replaced = []
        self.ctx.stream_end()
        res = [self.ctx.get_layer(lid) for lid in self.layer_ids]   # synchronises: the borrowed tensors are free
        self._keep = []
        self._pending = []
        return res

    # -- running the model in a low-precision configuration --------------------
    @contextlib.contextmanager
    def quantised(self, fmt_of_layer, amax_x=None):
        """Inside this block layer i (index into ``modules``) runs with its input and
        weight rounded to format ``fmt_of_layer[i]`` (0 leaves it alone).
        ``amax_x[i]`` is the static amax of the layer's input (measured per call if
        absent); the weight's amax is always measured."""
        saved, handles = [], []
        for idx, (_, m) in enumerate(self.modules):
            fmt = fmt_of_layer[idx]
            if not fmt:
                continue
            if isinstance(m, BatchedMatmul):   # both inputs rounded, each with its own measured amax

                def pre2(module, inputs, fmt=fmt):
                    outs = []
                    for x in inputs:
                        x = x.contiguous()
                        out = torch.empty_like(x)
                        self.ctx.fake_quant(ampq.torch_dtype_code(x), fmt, x.data_ptr(), x.numel(), -1.0, out.data_ptr())
                        self._keep.append(x)
                        outs.append(out)
                    return tuple(outs)

                handles.append(m.register_forward_pre_hook(pre2))
                continue
            w = m.weight.data
            saved.append((m, w.clone()))
            self.ctx.fake_quant(ampq.torch_dtype_code(w), fmt, w.data_ptr(), w.numel(), -1.0, w.data_ptr())

            def pre(module, inputs, fmt=fmt, a=(-1.0 if amax_x is None else float(amax_x[idx]))):
                x = inputs[0].contiguous()
                out = torch.empty_like(x)
                self.ctx.fake_quant(ampq.torch_dtype_code(x), fmt, x.data_ptr(), x.numel(), a, out.data_ptr())
                self._keep.append(x)
                return (out,) + tuple(inputs[1:])

            handles.append(m.register_forward_pre_hook(pre))
        try:
            yield
        finally:
            torch.cuda.current_stream().synchronize()
            for h in handles:
                h.remove()
            for m, w in saved:
                m.weight.data.copy_(w)
            if not self._same_stream():
                torch.cuda.ExternalStream(self.ctx.stream).synchronize()
            self._keep = []
