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


class Tied(torch.nn.Module):
    """An embedding, a layer and a head, which shares the embedding's weight or has a copy of it."""

    def __init__(self, dec, tied):
        super().__init__()
        torch.manual_seed(5)
        self.embed = dec.ScaledEmbedding(97, 64, device="cuda")
        self.layer, self.head = torch.nn.Linear(64, 64, device="cuda"), torch.nn.Linear(64, 97, bias=False, device="cuda")
        if tied:
            self.head.weight = self.embed.weight
        else:
            self.head.weight.data.copy_(self.embed.weight.data)

    def forward(self, tokens):
        return self.head(self.layer(self.embed(tokens)).tanh())


def test_tied_embedding(ampq, dec):
    """A head whose weight is the embedding's diverges as one with a copy of it, and both stay as they were."""
    from paper_2505_13060_b200 import hooks

    ctx = ampq.Context(0, torch.cuda.current_stream().cuda_stream)
    ctx.set_formats([0, 1])
    tokens = torch.randint(0, 97, (3, 20), generator=torch.Generator().manual_seed(1)).cuda()
    out = []
    for tied in (True, False):
        net = Tied(dec, tied)
        before = [t.detach().clone() for t in net.parameters()]
        cal = hooks.Calibrator(ctx, net, 1)
        out.append(cal.divergence(lambda: net(tokens), [0, 1], top=97))
        assert all(torch.equal(a, b) for a, b in zip(before, net.parameters())) and (net.head.weight is net.embed.weight) == tied
    assert torch.equal(*out) and float(out[0].mean()) > 0
    ctx.destroy()


def test_refused_in_the_middle(ampq, dec):
    """A format that the context does not list, and weights of a type that is not rounded: the model stays as it was."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        before = [t.detach().clone() for t in net.parameters()]
        cal = hooks.Calibrator(ctx, net, 1)
        for formats in ([1] * 12 + [2], [1] * 3 + [2] + [1] * 9):
            with pytest.raises(ampq.AmpqError):
                cal.divergence(lambda: net(tokens), formats)
            assert all(torch.equal(a, b) for a, b in zip(before, net.parameters())) and not any(m._forward_pre_hooks for m in net.modules())
        want = net(tokens)
        cal.divergence(lambda: net(tokens), [1] * 13)
        assert torch.equal(net(tokens), want)
