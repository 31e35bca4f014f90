"""Arguments of the decoder's operators that are looked at before anything runs: nothing here needs a GPU."""
import pytest
import torch


@pytest.fixture
def dec(ampq, monkeypatch):
    from paper_2505_13060_b200 import decoder

    monkeypatch.setattr(decoder, "_same_device", lambda *a: None)
    return decoder


def rows_of(dec, positions, leading, tokens):
    """The positions [batch, tokens] that the kernel would read."""
    batch = 1
    for d in leading:
        batch *= d
    cos, sin = dec.rotary_table(50, 8, device="cpu")
    turn, held = dec._rotation(cos, sin, positions, batch, tokens, 0, torch.Size(leading))
    p, stride = held[2], turn[6]
    assert turn[4] == p.data_ptr()
    return torch.as_strided(p, (batch, tokens), (stride, 1), p.storage_offset())


@pytest.mark.parametrize("shape,leading", [((7,), (3,)), ((3, 7), (3,)), ((1, 7), (3,)), ((1, 7), (1,)), ((7,), ()), ((2, 3, 7), (2, 3)), ((1, 3, 7), (2, 3)),
                                           ((2, 1, 7), (2, 3)), ((1, 1, 7), (2, 3)), ((3, 7), (2, 3)), ((1, 7), (2, 3)), ((1, 7), (0,)), ((2, 3, 1), (2, 3)), ((1, 1), (4,))])
def test_positions_of_a_batch(dec, shape, leading):
    """Positions that hold for several of a batch, as models hand them on: [1, tokens] for a batch of any size."""
    tokens = shape[-1]
    p = torch.randint(0, 50, shape, generator=torch.Generator().manual_seed(0))
    want = p.expand(*leading, tokens).reshape(-1, tokens)
    assert torch.equal(rows_of(dec, p, leading, tokens), want)
    wide = torch.zeros(*shape[:-1], 2 * tokens, dtype=torch.int64)
    wide[..., ::2] = p
    assert torch.equal(rows_of(dec, wide[..., ::2], leading, tokens), want)


@pytest.mark.parametrize("shape,leading", [((2, 7), (3,)), ((1, 1, 7), (3,)), ((3, 1), (3,)), ((6,), (3,)), ((), (3,)), ((3, 2, 7), (2, 3)), ((2, 7), (2, 3)), ((1, 7), ())])
def test_positions_that_are_not_those_of_the_tokens(dec, shape, leading):
    with pytest.raises(ValueError, match="positions"):
        rows_of(dec, torch.zeros(shape, dtype=torch.int64), leading, 7)


def test_constants_that_want_a_gradient(dec):
    """Refused where their gradient would be dropped without a word, and only there."""
    x, cos, sin = torch.zeros(3, 2, 8), *dec.rotary_table(3, 8, device="cpu")
    lists = torch.zeros(9, 2, dtype=torch.int64), torch.zeros(9, 2, requires_grad=True)
    for call in (lambda: dec.head_norm(x, None, None, None, cos.requires_grad_(), sin.detach()), lambda: dec.head_norm(x, None, None, None, cos.detach(), sin.requires_grad_()),
                 lambda: dec.distill_loss(torch.zeros(9, 40), *lists)):
        with pytest.raises(ValueError, match="constant"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):   # what is wrong then is only that there is no GPU
            call()


def test_one_layout_of_the_heads(dec, ampq):
    """What a call packs is the structure field by field."""
    import ctypes as C

    from paper_2505_13060_b200.checkpoint import Packed

    out, x, gy = torch.zeros(2, 3, 4, 8), torch.zeros(2, 3, 6, 8)[:, :, :4], torch.zeros(2, 4, 3, 8).transpose(1, 2)
    rstd, w, gw = torch.zeros(2, 3, 4), torch.zeros(8), torch.zeros(8)
    p = object.__new__(Packed)
    p.codes, p.scales = torch.zeros(24, 32, dtype=torch.uint8), torch.zeros(24, 1, dtype=torch.uint8)
    want = ampq.Heads(heads=4, x=x.data_ptr(), x_batch=144, x_token=48, x_head=8, gy=gy.data_ptr(), gy_batch=96, gy_token=8, gy_head=24, out=out.data_ptr(), out_batch=96,
                      out_token=32, out_head=8, weight=w.data_ptr(), gweight=gw.data_ptr(), rstd=rstd.data_ptr(), codes=p.codes.data_ptr(), ld_codes=32,
                      scales=p.scales.data_ptr(), ld_scales=1)
    assert dec._side(out, rstd, w, x=x, gy=gy, gw=gw, kept=p) == bytes(want)
    none = ampq.Heads(heads=4, out=out.data_ptr(), out_batch=96, out_token=32, out_head=8, rstd=rstd.data_ptr())
    assert dec._side(out, rstd, None) == bytes(none) and C.sizeof(none) == 8 * len(none._fields_)
