"""Running a model in a low-precision configuration, with a context and streams that stand in for the GPU's: nothing here
needs one."""
import ctypes as C

import numpy as np
import pytest
import torch
import torch.nn.utils.prune


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
        self.log, self.stream, self.layers, self.device = log, stream, 0, 0

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
    monkeypatch.setattr(hooks.Calibrator, "_device_of", staticmethod(lambda x: x.device.index or 0), raising=False)
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


def test_shared_weights_are_rounded_for_their_layer_alone(setup):
    """An embedding that is tied to the head is looked up as it was, layers that share a weight have it in their own formats,
    and afterwards everything is as before."""
    make, _ = setup
    lookup, head, other, alone = torch.nn.Embedding(5, 4), torch.nn.Linear(4, 5, bias=False), torch.nn.Linear(4, 5, bias=False), torch.nn.Linear(4, 4)
    head.weight = other.weight = lookup.weight
    before = lookup.weight.detach().clone()
    net = torch.nn.ModuleList([lookup, head, other, alone])
    cal = make(net)
    with cal.quantised([1, 3, 0]):
        assert torch.equal(lookup(torch.arange(5)), before)
        assert torch.equal(head(torch.eye(4)), rounded(before, 1).t()) and torch.equal(other(torch.eye(4)), rounded(before, 3).t())
        assert not torch.equal(rounded(before, 1), rounded(before, 3))
    assert head.weight is other.weight is lookup.weight and isinstance(head.weight, torch.nn.Parameter) and torch.equal(lookup.weight, before)
    assert len(list(net.parameters())) == 3


def test_an_exception_leaves_the_model_as_it_was(setup):
    make, _ = setup
    net = torch.nn.Sequential(*(torch.nn.Linear(4, 4) for _ in range(3)))
    before, x = [p.detach().clone() for p in net.parameters()], torch.randn(2, 4)
    cal = make(net)

    def same():
        return all(torch.equal(a, b) for a, b in zip(before, net.parameters())) and not any(m._forward_pre_hooks for m in net)

    for formats, amax in (([1, 2], None), ([1, 2, -1], None), ([1, 2, 3], [1.0]), ([1, 2, 3], [1.0, 2.0, None])):
        with pytest.raises((ValueError, IndexError, TypeError)):
            with cal.quantised(formats, amax):
                pass
        assert same()
    with cal.quantised([1, 0, 3], [1.0, None, -1.0]), torch.no_grad():   # what is not rounded has no amax
        net(x)
    assert same()
    net[2].double()
    with pytest.raises((ValueError, KeyError, TypeError)):   # a weight of a type that is not rounded
        with cal.quantised([1, 2, 3]):
            pass
    net[2].float()
    assert same()
    with pytest.raises(KeyError):
        with cal.quantised([1, 2, 3]):
            net(x)
            raise KeyError
    assert same()


def test_weights_that_are_no_parameters(setup):
    """A buffer, a view of a wider tensor, a gradient through a rounded weight, and a weight that the module computes."""
    make, _ = setup
    wide = torch.randn(4, 9)
    copy = wide.clone()
    a, b = torch.nn.Linear(6, 4, bias=False), torch.nn.Linear(4, 3, bias=False)
    del a.weight
    a.register_buffer("weight", wide[:, :6])
    cal = make(torch.nn.Sequential(a, b))
    x = torch.round(torch.randn(2, 6))
    with cal.quantised([1, 2]):
        h = a(x)
        assert torch.equal(h, x @ rounded(copy[:, :6], 1).t())
        b(h).sum().backward()
    assert torch.equal(wide, copy) and a.weight.data_ptr() == wide.data_ptr()
    assert torch.allclose(b.weight.grad, rounded(h, 2).sum(0).expand(3, 4))
    for c in (torch.nn.utils.parametrizations.weight_norm(torch.nn.Linear(4, 4)), torch.nn.utils.prune.l1_unstructured(torch.nn.Linear(4, 4), "weight", 0.5)):
        with pytest.raises(ValueError, match="computes its weight"):
            with make(torch.nn.Sequential(c)).quantised([1]):
                pass


def test_divergence_refuses_before_the_second_pass(setup, monkeypatch):
    """What it cannot do with its arguments is said before the model runs, what it cannot do with the logits before it
    runs again; the model stays as it was."""
    from paper_2505_13060_b200 import decoder

    make, _ = setup
    net = torch.nn.Linear(4, 5)
    cal, calls, logits = make(net), [], [torch.zeros(2, 3000)]

    def forward():
        calls.append(1)
        return logits[0]

    for formats, more in (([], {}), ([1], dict(top=-1)), ([1], dict(temperature=0.0)), ([1], dict(temperature=2.0 ** 21)), ([1], dict(temperature=float("nan")))):
        with pytest.raises((ValueError, IndexError)):
            cal.divergence(forward, formats, **more)
    assert not calls
    with pytest.raises(ValueError, match="CUDA"):
        cal.divergence(forward, [1])
    monkeypatch.setattr(decoder, "_device_of", lambda t: 0)
    for bad, top, error in ((logits[0].half(), 64, TypeError), (logits[0], 1025, ValueError), (logits[0].sum(), 64, ValueError)):
        logits[0] = bad
        calls.clear()
        with pytest.raises(error):
            cal.divergence(forward, [1], top=top)
        assert len(calls) == 1
    assert not net._forward_pre_hooks
    assert decoder.list_length(torch.zeros(2, 301), 5000) == 301   # of all there are


def test_tensors_that_are_not_on_the_contexts_device(setup, monkeypatch):
    """Their addresses never reach the context: a model on the host, or on another GPU."""
    from paper_2505_13060_b200 import hooks

    make, log = setup
    net = torch.nn.Linear(4, 4)
    before = net.weight.detach().clone()
    for where in (-1, 1):
        monkeypatch.setattr(hooks.Calibrator, "_device_of", staticmethod(lambda x: where))
        with pytest.raises(ValueError, match="context on cuda:0"):
            with make(net).quantised([1]):
                pass
    assert not log.count("round") and torch.equal(net.weight, before)
    monkeypatch.undo()
    assert hooks.Calibrator._device_of(net.weight) == -1
