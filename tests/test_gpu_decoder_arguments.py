"""Forms of the arguments of the decoder's operators that mean the same."""
import pytest
import torch

from test_gpu_decoder import dec, randn  # noqa: F401 (dec is a fixture)

pytestmark = pytest.mark.gpu


def test_positions_of_a_batch(dec):
    """[1, tokens] for a batch of three, and for two dimensions in front: the same bits as one by one, in both passes."""
    cos, sin = dec.rotary_table(50, 64)
    at = torch.randint(0, 50, (1, 9), generator=torch.Generator().manual_seed(0)).cuda()
    q, k = randn((3, 9, 4, 64), torch.bfloat16, 1), randn((3, 9, 2, 64), torch.bfloat16, 2)
    want = dec.head_norm_forward(q, k, None, None, cos, sin, at.expand(3, 9).contiguous())
    got = dec.head_norm_forward(q, k, None, None, cos, sin, at)
    assert all(torch.equal(a, b) for a, b in zip(got[:4], want[:4]))
    back = [dec.head_norm_backward(q, k, q, k, want[2], want[3], None, None, cos, sin, p) for p in (at.expand(3, 9).contiguous(), at)]
    assert all(torch.equal(a, b) for a, b in zip(back[0][:2], back[1][:2]))
    five = dec.head_norm_forward(q[None], k[None], None, None, cos, sin, at)
    assert torch.equal(five[0][0], want[0])
    two = torch.randint(0, 50, (2, 1, 9), generator=torch.Generator().manual_seed(1)).cuda()
    x = randn((2, 3, 9, 4, 64), torch.float32, 3)
    assert torch.equal(dec.head_norm_forward(x, None, None, None, cos, sin, two)[0],
                       dec.head_norm_forward(x, None, None, None, cos, sin, two.expand(2, 3, 9).contiguous())[0])
