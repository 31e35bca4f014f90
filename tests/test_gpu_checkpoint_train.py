"""8-bit checkpoints as a model meets them: the differentiable linear layer and
norms, a small network trained a step through them, and a calibration whose
layers keep their inputs in 8 bits."""
import numpy as np
import pytest
import torch

import ckpt_reference as ref
from helpers import assert_close

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]
IDS = {torch.float32: "f32", torch.bfloat16: "bf16"}


@pytest.fixture(scope="module")
def ckpt(ampq):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2505_13060_b200 import checkpoint

    return checkpoint


def f64(t):
    return t.detach().double().cpu().numpy()


def decoded(x, fmt):
    v = f64(x).reshape(-1, x.shape[-1])
    return ref.unpack(*ref.pack(v, fmt), v.shape[1], fmt)


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_linear(ckpt, dtype, fmt):
    """gw is that of the decoded input, gx and gb are exact, and x is kept as 33/32 byte per element."""
    g = torch.Generator(device="cuda").manual_seed(fmt)
    x = torch.randn(3, 70, 200, device="cuda", generator=g).to(dtype).requires_grad_()
    w = (torch.randn(90, 200, device="cuda", generator=g) * 0.1).to(dtype).requires_grad_()
    b = torch.randn(90, device="cuda", generator=g).to(dtype).requires_grad_()
    gy = torch.randn(3, 70, 90, device="cuda", generator=g).to(dtype)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        y = ckpt.linear(x, w, b, fmt)
    assert torch.equal(y, torch.nn.functional.linear(x, w, b))
    assert not any(t.data_ptr() == x.data_ptr() for t in kept)
    assert sum(t.numel() * t.element_size() for t in kept if t.dtype == torch.uint8) == 210 * (224 + 7)
    y.backward(gy)
    xd, gd = decoded(x, fmt), f64(gy).reshape(-1, 90)
    want, size = gd.T @ xd, np.abs(gd).T @ np.abs(xd)
    h = HALF_STEP[dtype]
    assert (np.abs(f64(w.grad) - want) <= (2 * 210 + 8) * U * size + 1.01 * h * np.abs(want)).all()
    want = gd.sum(0)
    assert (np.abs(f64(b.grad) - want) <= 220 * U * np.abs(gd).sum(0) + 1.01 * h * np.abs(want)).all()
    assert torch.equal(x.grad, torch.matmul(gy, w.detach()))


def test_linear_parts(ckpt):
    """Frozen weights keep nothing of x, and each gradient can be asked for alone."""
    x, w, b = torch.randn(40, 64, device="cuda"), torch.randn(24, 64, device="cuda"), torch.randn(24, device="cuda")
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        y = ckpt.linear(x.clone().requires_grad_(), w, None)
    assert [t.dtype for t in kept] == [torch.float32]
    xg, wg, bg = x.clone().requires_grad_(), w.clone().requires_grad_(), b.clone().requires_grad_()
    ckpt.linear(xg, w, b).sum().backward()   # the gradient of a sum is one number expanded
    # a sum of n terms in fp32, whatever its order, is off by at most n * 2^-24 of the absolute sum
    assert bool(((xg.grad - w.double().sum(0)).abs() <= 24 * U * w.double().abs().sum(0)).all())
    ckpt.linear(x, wg, b).sum().backward()
    kept_x = ckpt.unpack(ckpt.pack(x), torch.float32).double()
    assert bool(((wg.grad - kept_x.sum(0)).abs() <= (2 * 40 + 8) * U * kept_x.abs().sum(0)).all())
    ckpt.linear(x, w, bg).sum().backward()
    assert torch.equal(bg.grad, torch.full_like(b, 40.0))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_norms(ckpt, kind, fmt):
    """Gradients through the differentiable norms are those of the plain calls."""
    from paper_2505_13060_b200 import binding

    x = torch.randn(5, 33, 136, device="cuda", dtype=torch.bfloat16).requires_grad_()
    w = torch.rand(136, device="cuda").requires_grad_()
    b = torch.rand(136, device="cuda").requires_grad_()
    gy = torch.randn(5, 33, 136, device="cuda", dtype=torch.bfloat16)
    code = binding.NORM_LAYER if kind == "layer" else binding.NORM_RMS
    y = ckpt.layer_norm(x, w, b, 1e-5, fmt) if kind == "layer" else ckpt.rms_norm(x, w, 1e-5, fmt)
    y.backward(gy)
    want, mean, rstd, p = ckpt.norm_forward(x.detach(), w.detach(), b.detach() if kind == "layer" else None, 1e-5, code, fmt)
    gx, gw, gb = ckpt.norm_backward(gy, p if fmt else x.detach(), mean, rstd, w.detach(), code)
    assert torch.equal(y, want) and torch.equal(x.grad, gx) and torch.equal(w.grad, gw) and y.shape == x.shape
    assert (b.grad is None) if kind == "rms" else torch.equal(b.grad, gb)
    # the values of torch's own norm, one rounding of a bf16 output apart
    own = torch.nn.functional.layer_norm(x.float(), (136,), w, b) if kind == "layer" else torch.nn.functional.rms_norm(x.float(), (136,), w, 1e-5)
    assert (y.float() - own).abs().max() <= 2.0 ** -8 * own.abs().max() * 1.01


class Block(torch.nn.Module):
    def __init__(self, c, rms):
        super().__init__()
        self.norm = torch.nn.RMSNorm(c) if rms else torch.nn.LayerNorm(c)
        self.up, self.down = torch.nn.Linear(c, 3 * c), torch.nn.Linear(3 * c, c, bias=False)

    def forward(self, x):
        return x + self.down(torch.nn.functional.gelu(self.up(self.norm(x))))


def model(seed, c=96, dtype=torch.float32):
    torch.manual_seed(seed)
    return torch.nn.Sequential(torch.nn.Linear(40, c), Block(c, False), Block(c, True), torch.nn.Linear(c, 1)).cuda().to(dtype)


@pytest.mark.parametrize("fmt", [1, 2])
def test_calibration_with_checkpoints(ampq, orc, fmt):
    """Sensitivities of every linear layer against the oracle, from the inputs and gradients of the same run captured
    from outside: the layer's input decoded by the reference, dL/dX as the layer's hook sees it, dL/dW formed in 64 bits."""
    from paper_2505_13060_b200 import hooks

    R, tokens = 3, 50
    net = model(5)
    net.requires_grad_(True)
    ctx = ampq.Context(0, torch.cuda.current_stream().cuda_stream)
    ctx.set_formats([0, 1])
    cal = hooks.Calibrator(ctx, net, R, checkpoint=fmt)
    cal.begin()
    seen = [{} for _ in cal.modules]
    handles = []
    for k, (_, m) in enumerate(cal.modules):
        handles.append(m.register_forward_hook(lambda mod, i, o, k=k: seen[k].setdefault("x", []).append(i[0].detach().clone())))
        handles.append(m.register_full_backward_hook(lambda mod, gi, go, k=k: (seen[k].setdefault("gx", []).append(None if gi[0] is None else gi[0].detach().clone()),
                                                                              seen[k].setdefault("gy", []).append(go[0].detach().clone()))[0] and None))
    batch = torch.randn(R, tokens, 40, device="cuda")
    for r in range(R):
        with cal.sample(r):
            net(batch[r]).square().mean().backward()
    res = cal.end()
    for h in handles:
        h.remove()
    assert not any("forward" in m.__dict__ for m in net.modules())
    for k, ((name, m), got) in enumerate(zip(cal.modules, res)):
        w = f64(m.weight)
        for r in range(R):
            x = decoded(seen[k]["x"][r], fmt)
            gy = f64(seen[k]["gy"][r]).reshape(len(x), -1)
            gx = gy @ w if seen[k]["gx"][r] is None else f64(seen[k]["gx"][r]).reshape(x.shape)
            want = ((x * gx) ** 2).sum() + ((w * (gy.T @ x)) ** 2).sum()
            # fp32 gradients: a product over n terms is off by about n * 2^-24 of its absolute sum, a few times its size here
            assert abs(got["s_per_sample"][r] - want) <= 1e-4 * want, (name, r)
        assert not got["d_meas"].any()
    # The last layer's dL/dY depends on no checkpoint.  A value off by at most u, half a step, has a square off by at
    # most 2u + u^2, and so has the sum over the layer's input.
    u = 2.0 ** -4 if fmt == 1 else 2.0 ** -3
    for r in range(R):
        x, gx = f64(seen[-1]["x"][r]), f64(seen[-1]["gy"][r]) @ f64(cal.modules[-1][1].weight)
        a, b = ((x * gx) ** 2).sum(), ((decoded(seen[-1]["x"][r], fmt) * gx) ** 2).sum()
        assert abs(a - b) <= (2 * u + u * u) * a
    # the same model calibrates without checkpoints afterwards
    ctx.set_measured(True)
    plain = hooks.Calibrator(ctx, net, 1)
    plain.begin()
    with plain.sample(0):
        net(batch[0]).square().mean().backward()
    assert all(f["s_mean"] > 0 and f["d_meas"][1] > 0 for f in plain.end())
    ctx.destroy()


def test_training_steps_graph(ckpt):
    """A training step of norm, linear, norm, linear through the checkpoints, captured once and replayed: the same
    gradients as run eagerly on the same inputs."""
    dtype = torch.bfloat16
    torch.manual_seed(1)
    w = [torch.rand(128, device="cuda").to(dtype), (torch.randn(320, 128, device="cuda") * 0.1).to(dtype), torch.rand(320, device="cuda").to(dtype),
         torch.rand(320, device="cuda").to(dtype), (torch.randn(64, 320, device="cuda") * 0.1).to(dtype)]
    x = torch.randn(300, 128, device="cuda").to(dtype)

    def step():
        leaves = [t.detach().requires_grad_() for t in w]
        h = ckpt.linear(ckpt.rms_norm(x, leaves[0]), leaves[1])
        y = ckpt.linear(ckpt.layer_norm(torch.nn.functional.silu(h), leaves[2], leaves[3]), leaves[4], fmt=2)
        return torch.autograd.grad(y.float().square().sum(), leaves)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (3, 4):
        x.copy_(torch.randn(300, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
