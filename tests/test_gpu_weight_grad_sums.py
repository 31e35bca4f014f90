"""Sums of the weight gradient over very many tokens, against sums in 64 bits."""
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


@pytest.mark.parametrize("outs,cols", [(1280, 2048), (1280, 1024)], ids=["pairs", "single"])
def test_bf16_sums_of_one_sign(ckpt, outs, cols):
    """2^20 tokens of one sign in bf16.  The tensor core cuts each addition by up to 2^-23 of the partial sum, always the
    same way: over all the tokens, which one tile takes here (there are too many tiles to share the token axis), that is
    more than half a step of bf16 (5e-3).  Taken out every 4096 tokens: at most 4096 cut additions in a run, 256 rounded ones
    that join the runs (2^-24 each), and half a step, 2^-8, at the end."""
    rows = 2 ** 20
    g = torch.Generator(device="cuda").manual_seed(cols)
    gy = torch.empty(rows, outs, dtype=torch.bfloat16, device="cuda").uniform_(1.0, 2.0, generator=g)
    gy *= torch.empty(outs, dtype=torch.bfloat16, device="cuda").uniform_(1.0, 2.0, generator=g)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").uniform_(1.0, 2.0, generator=g)
    p = ckpt.pack(x)
    del x
    gw, _ = ckpt.weight_grad(p, gy)
    some = ckpt.Packed(p.codes[:, :64], p.scales[:, :2], 64, p.fmt)
    want = torch.matmul(gy[:, :64].double().T, ckpt.unpack(some, torch.float32).double())
    off = (gw[0, :64, :64].double() - want).abs() / want
    assert float(off.max()) <= 2.0 ** -8 + 1.01 * (4096 * 2 * U + 256 * U)


@pytest.mark.parametrize("rows", [200, 300], ids=["small", "large"])
@pytest.mark.parametrize("exponent", [-100, -112, -120, -126, -140])
def test_fp32_gradients_near_the_smallest(ckpt, rows, exponent):
    """fp32 gradients are read to 24 significant bits down to 2^-110 and below that, where the products run on the tensor
    cores, to 2^-133 (bf16's last bit): what is cut off a gradient times |x|, on top of the bound of the sum itself and of an
    fp32 result, whose own last bit is 2^-149."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    gy = (torch.randn(rows, 520, device="cuda", generator=g).double() * 2.0 ** exponent).float()
    p = ckpt.pack(torch.randn(rows, 512, device="cuda", generator=g))
    x = ckpt.unpack(p, torch.float32).double()
    gw, gb = ckpt.weight_grad(p, gy, bias=True)
    want, size = gy.double().T @ x, gy.double().abs().T @ x.abs()
    tol = (2 * rows + 8) * U * size + U * want.abs() + 2.0 ** -150 * rows
    if rows > 256 and exponent < -100:
        tol += 2.0 ** -133 * x.abs().sum(0)
    assert bool(((gw[0].double() - want).abs() <= tol).all())
    assert bool(((gb[0].double() - gy.double().sum(0)).abs() <= rows * U * gy.double().abs().sum(0)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("samples,rows,cols,outs", [(2, 128, 256, 256), (3, 997, 1031, 2053), (1, 9000, 300, 520), (1, 6000, 4096, 2560), (2, 4096, 2048, 4096)])
def test_results_repeat_themselves(ckpt, dtype, samples, rows, cols, outs):
    """The same bits every time, with other work in between: sums are added in an order fixed by the sizes."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    p = ckpt.pack(torch.randn(samples * rows, cols, device="cuda", generator=g).to(dtype))
    gy = torch.randn(samples * rows, outs, device="cuda", generator=g).to(dtype)
    first = ckpt.weight_grad(p, gy, samples=samples, bias=True)
    for _ in range(8):
        ckpt.weight_grad(p, gy + 1, samples=samples, bias=True)
        again = ckpt.weight_grad(p, gy, samples=samples, bias=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("outs,cols", [(2050, 1290), (1290, 1030)], ids=["pairs", "single"])
@pytest.mark.parametrize("rows", [4096, 4097, 8193])
def test_around_the_length_of_a_run(ckpt, dtype, outs, cols, rows):
    """One run of tokens, a second one of a single token, a third: every output, odd widths.  A sum of n terms is off by at
    most 2 n * 2^-24 of its absolute sum (cut additions), and half a step at the end."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    p = ckpt.pack(torch.randn(rows, cols, device="cuda", generator=g).to(dtype))
    gy = torch.randn(rows, outs, device="cuda", generator=g).to(dtype)
    x = ckpt.unpack(p, torch.float32).double()
    gw, gb = ckpt.weight_grad(p, gy, bias=True)
    want, size = gy.double().T @ x, gy.double().abs().T @ x.abs()
    half = U if dtype == torch.float32 else 2.0 ** -8
    assert bool(((gw[0].double() - want).abs() <= 2 * rows * U * size + 1.01 * half * want.abs()).all())
    want, size = gy.double().sum(0), gy.double().abs().sum(0)
    assert bool(((gb[0].double() - want).abs() <= rows * U * size + 1.01 * half * want.abs()).all())
