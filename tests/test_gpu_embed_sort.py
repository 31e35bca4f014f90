"""The embedding gradient's sort of many tokens: an odd and an even number of passes, whose result lies in either pair of
buffers, tables of any size around the digits' borders, and tokens that are no row among them."""
import pytest
import torch

from test_gpu_decoder import check_embed_grad, dec, randn  # noqa: F401 (dec is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,cols", [(255, 40), (256, 40), (257, 33), (32000, 24), (65535, 8), (65536, 8), (2 ** 24 - 1, 1), (2 ** 24, 1), (2 ** 24 + 1, 2)])
def test_passes(dec, vocab, cols):
    g = torch.Generator().manual_seed(vocab % 1000)
    tokens = torch.randint(0, vocab, (9001,), generator=g)
    tokens[::3] = torch.randint(max(0, vocab - 5), vocab, (3001,), generator=g)   # runs at the table's end
    check_embed_grad(dec, tokens.cuda(), randn((9001, cols), torch.float32, 1), vocab, 1.0)
    if vocab < 100000:
        check_embed_grad(dec, tokens.cuda(), randn((9001, cols), torch.bfloat16, 2), vocab, 0.5, vocab - 1, torch.int32)
        outside = tokens.clone()
        outside[5::7] = -1
        outside[6::7] = vocab
        gy = randn((9001, cols), torch.float32, 3)
        inside = torch.where((outside >= 0) & (outside < vocab), outside, 0)
        keep = ((outside >= 0) & (outside < vocab)).cuda()
        got = dec.embed_backward(outside.cuda(), gy, vocab)
        want = torch.zeros(vocab, cols, dtype=torch.float64, device="cuda").index_add_(0, inside.cuda(), gy.double() * keep[:, None])
        size = torch.zeros(vocab, cols, dtype=torch.float64, device="cuda").index_add_(0, inside.cuda(), gy.double().abs() * keep[:, None])
        # at most 9001 terms of a row are added in fp32, and the sum is rounded once
        assert bool(((got.double() - want).abs() <= 9003 * 2.0 ** -24 * size).all())
