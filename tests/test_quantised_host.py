"""Running a model in a low-precision configuration, with a context and streams that stand in for the GPU's: nothing here
needs one."""
import ctypes as C

import numpy as np
import pytest
import torch


class Stream:
    def __init__(self, log, name, handle):
        self.log, self.name, self.cuda_stream = log, name, handle

    def wait_stream(self, other):
        self.log.append("%s waits for %s" % (self.name, other.name))

    def synchronize(self):
        self.log.append("%s done" % self.name)


class Context:
    """Rounds fp32 values to multiples of 2^-fmt; -1 is a format that it does not list."""

    def __init__(self, log, stream):
        self.log, self.stream, self.layers = log, stream, 0

    def register_layer(self, kind, name, R):
        self.layers += 1
        return self.layers - 1

    def fake_quant(self, code, fmt, values, numel, amax, out):
        if fmt < 0:
            raise ValueError("format is not listed")
        self.log.append("round")
        x, y = (np.ctypeslib.as_array(C.cast(p, C.POINTER(C.c_float)), (numel,)) for p in (values, out))
        y[:] = np.round(x * 2.0 ** fmt) * 2.0 ** -fmt


def rounded(w, fmt):
    return torch.round(w.detach() * 2.0 ** fmt) * 2.0 ** -fmt


@pytest.fixture
def setup(monkeypatch):
    """A function of the model and the context's stream that makes a calibrator; and the log of what happened in order.
    Torch's current stream is 7."""
    from paper_2505_13060_b200 import hooks

    log = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(log, "torch", 7))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *a: Stream(log, "context", handle))
    return lambda model, stream=7: hooks.Calibrator(Context(log, stream), model, 1), log


def test_rounding_is_ordered_between_two_streams(setup):
    """What the context's stream rounds was made on torch's, and torch's reads the result: a wait in either direction around
    each rounding, of weights, of inputs and of both operands of a product.  On one stream there is none."""
    from paper_2505_13060_b200 import hooks

    make, log = setup

    class Net(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.a, self.mm = torch.nn.Linear(4, 4), hooks.BatchedMatmul()

        def forward(self, x):
            return self.mm(self.a(x), x.t())

    x = torch.randn(4, 4)
    for stream, once in ((9, ["context waits for torch", "round", "torch waits for context"]), (7, ["round"])):
        cal = make(Net(), stream)
        log.clear()
        with cal.quantised([2, 3]), torch.no_grad():
            assert log == once
            cal.model(x)
            assert log == 4 * once
