"""A calibration with 8-bit checkpoints runs the model it is given: the same forward pass but for the norms' last rounding,
every layer scored or the call refused, and model and context left as they were."""
import contextlib

import pytest
import torch

import ckpt_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hooks(ampq):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2505_13060_b200 import hooks

    return hooks


@pytest.fixture
def ctx(ampq):
    c = ampq.Context(0, torch.cuda.current_stream().cuda_stream)
    c.set_formats([0, 1])
    yield c
    c.destroy()


@contextlib.contextmanager
def one_sample(hooks, ctx, net, fmt=1):
    cal = hooks.Calibrator(ctx, net, 1, checkpoint=fmt)
    cal.begin()
    with cal.sample(0):
        yield cal
    cal.result = cal.end()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("affine", [True, False])
def test_rms_norm_of_default_eps(hooks, ctx, dtype, affine):
    """torch computes an RMSNorm without eps in fp32 with fp32's eps, whatever the input's type.  Values around 0.01 show
    which eps was used: bf16's own is as large as their square's root.  Both sides round an fp32 result once, off by half a
    step each; the fp32 results themselves agree to far less than a hundredth of a bf16 step, and to 2^-20 in fp32."""
    torch.manual_seed(1)
    norm = torch.nn.RMSNorm(192, elementwise_affine=affine).cuda().to(dtype)
    net = torch.nn.Sequential(norm, torch.nn.Linear(192, 8)).cuda().to(dtype)
    x = (torch.randn(40, 192, device="cuda") * 0.01).to(dtype)
    want = norm(x).double()
    with one_sample(hooks, ctx, net):
        got = norm(x).double()
        net(x).float().square().sum().backward()
    step = 2.0 ** -7 * 1.01 if dtype == torch.bfloat16 else 2.0 ** -20
    assert bool(((got - want).abs() <= step * want.abs()).all())


class Norm2d(torch.nn.LayerNorm):
    """A norm over the channels of [batch, channels, ...]."""

    def forward(self, x):
        return super().forward(x.transpose(1, -1)).transpose(1, -1)


class Doubled(torch.nn.Linear):
    """A linear layer with something beside its product."""

    def forward(self, x):
        return 2.0 * super().forward(x) + x.sum()


class Shifted(torch.nn.RMSNorm):
    def forward(self, x):
        return super().forward(x + 1.0)


@pytest.mark.parametrize("which", ["norm", "linear", "rms", "wrapped"])
def test_modules_with_a_forward_of_their_own(hooks, ctx, which):
    """Subclasses that do more than their base, and modules that somebody has wrapped already, run as they are; their
    linear layers are scored all the same."""
    torch.manual_seed(2)
    net = torch.nn.Sequential(Doubled(24, 24) if which == "linear" else torch.nn.Linear(24, 24),
                              {"norm": Norm2d(6), "rms": Shifted(24)}.get(which, torch.nn.LayerNorm(24)), torch.nn.Linear(24, 8)).cuda()
    if which == "wrapped":
        plain = net[0].forward
        net[0].forward = lambda x: plain(x) * 3.0
        mine = net[0].forward
    x = torch.randn(2, 6, 24, device="cuda")
    want = net(x).detach()
    with one_sample(hooks, ctx, net) as cal:
        y = net(x)
        y.square().sum().backward()
    # a norm of the library instead of torch's: some roundings of fp32 apart
    assert bool(((y - want).abs() <= 1e-5 * want.abs().max()).all())
    assert len(cal.result) == 2 and all(r["s_mean"] > 0 for r in cal.result)
    assert net[0].__dict__.get("forward") is (mine if which == "wrapped" else None)


def test_arguments_by_name(hooks, ctx):
    """Linear and LayerNorm call their argument `input`, RMSNorm `x`: all three can be called by name."""
    lin, ln, rms = torch.nn.Linear(32, 32).cuda(), torch.nn.LayerNorm(32).cuda(), torch.nn.RMSNorm(32).cuda()
    net = torch.nn.ModuleList([lin, ln, rms])
    x = torch.randn(5, 32, device="cuda")
    with one_sample(hooks, ctx, net) as cal:
        rms(x=ln(input=lin(input=x))).square().sum().backward()
    assert cal.result[0]["s_mean"] > 0


def test_types_that_cannot_be_kept_are_refused(hooks, ctx):
    """A layer that cannot be scored raises, as it does without checkpoints; it is not left out of the result silently."""
    net = torch.nn.Sequential(torch.nn.Linear(32, 8)).cuda().half()
    cal = hooks.Calibrator(ctx, net, 1, checkpoint=1)
    cal.begin()
    with pytest.raises(TypeError), cal.sample(0):
        net(torch.randn(4, 32, device="cuda").half()).float().square().sum().backward()
    cal.end()


def test_norms_that_the_library_does_not_have_run_plain(hooks, ctx):
    """fp16 parameters and inputs of another width: what torch does, its own error included."""
    ln = torch.nn.LayerNorm(32, elementwise_affine=False).cuda()
    net = torch.nn.ModuleList([ln, torch.nn.LayerNorm(32).cuda().half(), torch.nn.Linear(4, 4).cuda()])
    x = torch.randn(3, 32, device="cuda")
    with one_sample(hooks, ctx, net):
        with pytest.raises(RuntimeError):
            ln(torch.randn(3, 64, device="cuda"))
        assert torch.equal(net[1](x.half()), torch.nn.functional.layer_norm(x.half(), (32,), net[1].weight, net[1].bias))


def test_a_layer_that_runs_twice_is_refused(hooks, ctx):
    """One sample of a layer has one pair of operands: a layer that is used twice raises, as without checkpoints, instead of
    keeping the last use only."""
    lin = torch.nn.Linear(16, 16).cuda()
    for fmt in (0, 1):
        cal = hooks.Calibrator(ctx, lin, 1, checkpoint=fmt)
        cal.begin()
        with pytest.raises((KeyError, RuntimeError)), cal.sample(0):
            lin(lin(torch.randn(4, 16, device="cuda"))).square().sum().backward()
        with cal.sample(0):   # the sample again, used once
            lin(torch.randn(4, 16, device="cuda")).square().sum().backward()
        assert cal.end()[0]["s_mean"] > 0


def scored(cal, net, x, r=0):
    with cal.sample(r):
        net(x).square().sum().backward()


@pytest.mark.parametrize("how", ["ended", "raised", "dropped", "off"])
def test_the_context_and_the_model_are_left_as_they_were(hooks, ctx, how):
    """After a calibration with checkpoints the context scores the terms it scored before, also when a sample raised and
    when the calibration was dropped for another one."""
    net = torch.nn.Sequential(torch.nn.Linear(24, 24), torch.nn.LayerNorm(24), torch.nn.Linear(24, 8)).cuda()
    x = torch.randn(10, 24, device="cuda")
    if how == "off":
        ctx.set_measured(False)
    cal = hooks.Calibrator(ctx, net, 1, checkpoint=1)
    cal.begin()
    if how in ("raised", "dropped"):
        with pytest.raises(ZeroDivisionError), cal.sample(0):
            net(x)
            1 / 0
        assert not any("forward" in m.__dict__ for m in net.modules())
    if how == "raised":
        cal.begin()
    if how != "dropped":
        scored(cal, net, x)
        assert cal.end()[0]["s_mean"] > 0
        assert not any("forward" in m.__dict__ for m in net.modules())
    plain = hooks.Calibrator(ctx, net, 1)
    plain.begin()
    scored(plain, net, x)
    got = plain.end()[-2 if how != "dropped" else -1]
    assert (got["d_meas"][1] > 0) == (how != "off")


def test_what_a_sample_keeps(hooks, ctx):
    """On torch's own stream nothing of a layer outlives its backward step: the peak of a sample is its packed inputs (33/64
    of them in bf16) and what one layer needs, not every layer's decoded input and gradients."""
    tokens, c, layers = 4096, 2048, 24
    net = torch.nn.Sequential(*[torch.nn.Linear(c, c, bias=False) for _ in range(layers)]).cuda().bfloat16()
    x = torch.randn(tokens, c, device="cuda").bfloat16()
    full = x.numel() * 2
    peak = {}
    for fmt in (0, 1):
        cal = hooks.Calibrator(ctx, net, 2, checkpoint=fmt)
        cal.begin()
        scored(cal, net, x, 0)   # the parameters' gradients exist from here on
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        scored(cal, net, x, 1)
        torch.cuda.synchronize()
        peak[fmt] = (torch.cuda.max_memory_allocated() - before) / full
        cal.end()
    print("peak of a sample in inputs of a layer:", peak)
    assert peak[1] <= layers * 33 / 64 + 8
    assert peak[0] <= layers + 8


def test_autocast(hooks, ctx):
    """Under autocast the layers compute in bf16 from fp32 parameters, and are scored on what their product reads."""
    torch.manual_seed(3)
    net = torch.nn.Sequential(torch.nn.Linear(40, 32), torch.nn.LayerNorm(32), torch.nn.Linear(32, 8)).cuda()
    x = torch.randn(20, 40, device="cuda")
    with torch.autocast("cuda", torch.bfloat16):
        want = net(x).detach()
    with one_sample(hooks, ctx, net) as cal:
        with torch.autocast("cuda", torch.bfloat16):
            y = net(x)
            loss = y.float().square().sum()
        loss.backward()
    assert y.dtype == want.dtype and torch.equal(y, want)   # the norm is torch's own under autocast
    assert net[0].weight.grad.dtype == torch.float32 and bool(net[0].weight.grad.abs().sum() > 0)
    g = (2.0 * y.detach().double()).bfloat16().double()
    w = net[2].weight.detach().bfloat16().double()
    kept = net[1](torch.nn.functional.linear(x.bfloat16(), net[0].weight.bfloat16(), net[0].bias.bfloat16()).float()).detach().bfloat16().double()
    v = torch.tensor(ref.unpack(*ref.pack(kept.cpu().numpy(), 1), 32, 1), device="cuda")
    s = ((v * (g @ w)).square().sum() + (w * (g.T @ v)).square().sum()).item()
    # bf16 operands and gradients, each rounded by at most 2^-8: their products by 2 * 2^-8, the squares by twice that
    assert abs(cal.result[1]["s_mean"] - s) <= 0.02 * s


def test_results_stay_after_the_end(hooks, ctx):
    """Group costs and selections work on what was scored, as after any pass; the context's setting comes back with the next
    one, bound or streamed."""
    net = torch.nn.Linear(24, 8).cuda()
    x = torch.randn(10, 24, device="cuda")
    with one_sample(hooks, ctx, net) as cal:
        net(x).square().sum().backward()
    lid = cal.layer_ids[0]
    assert ctx.get_layer(lid)["s_mean"] == cal.result[0]["s_mean"] > 0
    g = torch.randn(10, 24, device="cuda")
    gw = torch.randn(8, 24, device="cuda")
    ctx.bind_operand(lid, 0, 0, x.data_ptr(), x.numel(), True, g.data_ptr(), x.numel())
    ctx.bind_operand(lid, 1, 0, net.weight.data_ptr(), gw.numel(), False, gw.data_ptr(), gw.numel())
    ctx.score()
    assert ctx.get_layer(lid)["d_meas"][1] > 0


@pytest.mark.parametrize("fmt", [0, 1])
def test_begin_again_after_a_sample_that_raised(hooks, ctx, fmt):
    """The hooks of the pass that was left are gone: each layer is seen once."""
    net = torch.nn.Sequential(torch.nn.Linear(24, 24), torch.nn.LayerNorm(24), torch.nn.Linear(24, 8)).cuda()
    x = torch.randn(10, 24, device="cuda")
    cal = hooks.Calibrator(ctx, net, 1, checkpoint=fmt)
    cal.begin()
    with pytest.raises(ZeroDivisionError), cal.sample(0):
        net(x)
        1 / 0
    cal.begin()
    scored(cal, net, x)
    assert all(r["s_mean"] > 0 for r in cal.end())
    assert not any(m._forward_hooks or m._backward_hooks for m in net.modules())


def test_a_context_on_a_stream_of_its_own(hooks, ampq):
    """The same sensitivities as on torch's stream, over more samples than are held at a time."""
    torch.manual_seed(4)
    net = torch.nn.Sequential(torch.nn.Linear(64, 256), torch.nn.LayerNorm(256), torch.nn.Linear(256, 64), torch.nn.RMSNorm(64), torch.nn.Linear(64, 8)).cuda().bfloat16()
    x = torch.randn(6, 500, 64, device="cuda").bfloat16()
    got = []
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        c = ampq.Context(0, stream.cuda_stream)
        c.set_formats([0, 1])
        cal = hooks.Calibrator(c, net, 6, checkpoint=1)
        cal.begin()
        for r in range(6):
            scored(cal, net, x[r], r)
        got.append([list(res["s_per_sample"]) for res in cal.end()])
        c.destroy()
    assert got[0] == got[1] and all(s > 0 for layer in got[0] for s in layer)
