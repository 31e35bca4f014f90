"""Edges of the checkpointed functions and norms: autocast, parameters of other types and shapes, rows without columns."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ckpt(ampq):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2505_13060_b200 import checkpoint

    return checkpoint


def test_linear_under_autocast(ckpt):
    """As torch's linear: operands cast to autocast's type, gradients in the parameters' own."""
    x, w, b = (torch.randn(*s, device="cuda").requires_grad_() for s in ((50, 72), (40, 72), (40,)))
    gy = torch.randn(50, 40, device="cuda").bfloat16()
    with torch.autocast("cuda", torch.bfloat16):
        y = ckpt.linear(x, w, b)
        want = torch.nn.functional.linear(x, w, b)
    assert y.dtype == torch.bfloat16 and torch.equal(y, want)
    y.backward(gy)
    cast = [t.detach().bfloat16().requires_grad_() for t in (x, w, b)]
    ckpt.linear(*cast).backward(gy)
    for t, c in zip((x, w, b), cast):
        assert t.grad.dtype == torch.float32 and torch.equal(t.grad, c.grad.float())


def test_linear_under_autocast_to_fp16_is_refused(ckpt):
    x, w = torch.randn(50, 72, device="cuda"), torch.randn(40, 72, device="cuda").requires_grad_()
    with torch.autocast("cuda", torch.float16), pytest.raises(TypeError):
        ckpt.linear(x, w)


def test_linear_of_two_types_is_refused(ckpt):
    """In the forward pass, by torch's own product."""
    with pytest.raises(RuntimeError):
        ckpt.linear(torch.randn(4, 32, device="cuda"), torch.randn(8, 32, device="cuda").bfloat16().requires_grad_())


@pytest.mark.parametrize("fmt", [0, 1])
def test_bias_without_weight(ckpt, fmt):
    """The bias's gradient comes in the bias's type, rounded to that alone: 300 additions in fp32."""
    x = torch.randn(300, 64, device="cuda").bfloat16()
    b = torch.randn(64, device="cuda").requires_grad_()
    gy = torch.randn(300, 64, device="cuda").bfloat16()
    ckpt.layer_norm(x, None, b, 1e-5, fmt).backward(gy)
    want = gy.double().sum(0)
    assert bool(((b.grad.double() - want).abs() <= 300 * U * gy.double().abs().sum(0)).all())


@pytest.mark.parametrize("fmt", [0, 1])
def test_parameters_of_more_dimensions(ckpt, fmt):
    """[1, C] parameters get gradients of their own shape."""
    x, gy = torch.randn(30, 64, device="cuda"), torch.randn(30, 64, device="cuda")
    w, b = torch.rand(1, 64, device="cuda").requires_grad_(), torch.rand(1, 64, device="cuda").requires_grad_()
    ckpt.layer_norm(x, w, b, 1e-5, fmt).backward(gy)
    v, c = w.detach()[0].clone().requires_grad_(), b.detach()[0].clone().requires_grad_()
    ckpt.layer_norm(x, v, c, 1e-5, fmt).backward(gy)
    assert torch.equal(w.grad[0], v.grad) and torch.equal(b.grad[0], c.grad)


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
def test_rows_without_columns_have_no_statistics(ampq, ckpt, kind, fmt):
    """The mean of nothing is NaN, and so is what follows from it; nothing is left unwritten."""
    mean, rstd = torch.full((7,), 3.0, device="cuda"), torch.full((7,), 3.0, device="cuda")
    rc = ampq.lib().ampq_norm_forward(0, torch.cuda.current_stream().cuda_stream, kind, 0, 0, fmt, 0, 0, 5, 0, 0, 0, 1e-5, 0, 0,
                                      mean.data_ptr() if kind == 0 else 0, rstd.data_ptr(), 0, 0, 0, 0)
    assert rc == 0
    assert bool(torch.isnan(rstd[:5]).all()) and bool((rstd[5:] == 3.0).all())
    if kind == 0:
        assert bool(torch.isnan(mean[:5]).all()) and bool((mean[5:] == 3.0).all())
    y, mean, rstd, p = ckpt.norm_forward(torch.empty(2, 3, 0, device="cuda"), None, None, 1e-5, kind, fmt)
    assert y.shape == (2, 3, 0) and bool(torch.isnan(rstd).all()) and (mean is None or bool(torch.isnan(mean).all()))
