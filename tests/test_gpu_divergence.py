"""Divergence of a low-precision configuration of a model on the GPU: a context on a stream of its own, shared weights, and
what is refused."""
import pytest
import torch

from test_gpu_decoder_train import a_decoder, dec  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def test_context_on_a_stream_of_its_own(ampq, dec):
    """The same bits as with a context on torch's stream, the model and the next call's result among them."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        forward = lambda: net(tokens)
        before = [t.detach().clone() for t in net.parameters()]
        want = hooks.Calibrator(ctx, net, 1).divergence(forward, [1] * 13)
        side = torch.cuda.Stream()
        other = ampq.Context(0, side.cuda_stream)
        other.set_formats([0, 1])
        cal = hooks.Calibrator(other, net, 1)
        for _ in range(10):
            assert torch.equal(cal.divergence(forward, [1] * 13), want)
            assert all(torch.equal(a, b) for a, b in zip(before, net.parameters()))
        other.destroy()
