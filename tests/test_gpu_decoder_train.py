"""The decoder's operators as a model meets them: differentiable forms, streams and graphs, far offsets, and a small
decoder that is calibrated and checked through them."""
import contextlib

import numpy as np
import pytest
import torch

import ckpt_reference as kept_ref
import decoder_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]
IDS = {torch.float32: "f32", torch.bfloat16: "bf16"}


@pytest.fixture(scope="module")
def dec(ampq):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2505_13060_b200 import decoder

    return decoder


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(shape, seed, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


# -- differentiable forms ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_embedding_gradients(dec, dtype):
    tokens = torch.randint(0, 30, (4, 50), generator=torch.Generator().manual_seed(0)).cuda()
    w = randn((30, 72), 1, dtype=dtype).requires_grad_()
    gy = randn((4, 50, 72), 2, dtype=dtype)
    y = dec.embedding(tokens, w, 1.5, padding_idx=3)
    assert torch.equal(y, dec.embed(tokens, w.detach(), 1.5))   # the padding row is read, it is not learnt
    y.backward(gy)
    assert torch.equal(w.grad, dec.embed_backward(tokens, gy, 30, 1.5, 3)) and not w.grad[3].any()
    with pytest.raises(ValueError, match="padding_idx"):
        dec.embedding(tokens, w, padding_idx=-1)
    m = dec.ScaledEmbedding(30, 72, 1.5, padding_idx=3, device="cuda", dtype=dtype)
    assert not m.weight[3].any()
    m.weight.data.copy_(w.detach())
    m(tokens).backward(gy)
    assert torch.equal(m.weight.grad, w.grad)
    with pytest.raises(ValueError):
        dec.ScaledEmbedding(30, 72, sparse=True)


def head_case(dec, dtype, seed=0, cols=64, rot=64, shape=(2, 20), hq=4, hk=2):
    cos, sin = dec.rotary_table(100, rot)
    positions = torch.randint(0, 100, shape, generator=torch.Generator().manual_seed(seed)).cuda()
    q, k = randn((*shape, hq, cols), seed + 1, dtype=dtype), randn((*shape, hk, cols), seed + 2, dtype=dtype)
    wq, wk = (1 + randn((cols,), seed + 3, 0.2)).to(dtype), (1 + randn((cols,), seed + 4, 0.2)).to(dtype)
    return [t.requires_grad_() for t in (q, k, wq, wk)], (cos, sin, positions)


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_head_norm_gradients(dec, dtype, fmt):
    """The gradients of the forward and backward calls, and what is kept of the inputs."""
    leaves, turn = head_case(dec, dtype)
    q, k, wq, wk = leaves
    gq, gk = randn(q.shape, 5, dtype=dtype), randn(k.shape, 6, dtype=dtype)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        yq, yk = dec.head_norm(*leaves, *turn, fmt=fmt)
    in_full = {q.data_ptr(), k.data_ptr()}
    assert sum(t.data_ptr() in in_full for t in kept) == (0 if fmt else 2)
    assert sum(t.numel() for t in kept if t.dtype == torch.uint8) == (2 * 20 * 6 * 66 if fmt else 0)
    torch.autograd.backward((yq, yk), (gq, gk))
    out = dec.head_norm_forward(*(t.detach() for t in leaves), *turn, fmt=fmt)
    assert torch.equal(out[0], yq) and torch.equal(out[1], yk)
    want = dec.head_norm_backward(gq, gk, *(out[4:] if fmt else (q.detach(), k.detach())), *out[2:4], wq.detach(), wk.detach(), *turn)
    for t, g in zip(leaves, want):
        assert torch.equal(t.grad, g) and t.grad.dtype == t.dtype


def test_head_norm_gradient_against_differences(dec):
    """The directional derivative of sum(y * g) along random directions, by central differences of the definition in 64
    bits: their own error is step^2 times the third derivative, about 1e-6 of the derivative here; the kernel's gradient is
    off by 2^-24 times a hundred operations of its sums, whose sizes are a few times their sum's root: 1e-4 of the norm of
    gradient times direction bounds both."""
    leaves, (cos, sin, positions) = head_case(dec, torch.float32, seed=20, cols=48, rot=16)
    q, k, wq, wk = leaves
    gq, gk = randn(q.shape, 25), randn(k.shape, 26)
    yq, yk = dec.head_norm(*leaves, cos, sin, positions, fmt=0)
    torch.autograd.backward((yq, yk), (gq, gk))
    at = positions.cpu().numpy()
    c, s = f64(cos)[at], f64(sin)[at]
    rng = np.random.default_rng(0)

    def f(q, k, wq, wk):
        return (ref.head_norm(q, wq, c, s, 16, 1e-5, False)[0] * f64(gq)).sum() + (ref.head_norm(k, wk, c, s, 16, 1e-5, False)[0] * f64(gk)).sum()

    x = [f64(t) for t in leaves]
    for i, t in enumerate(leaves):
        d = rng.standard_normal(x[i].shape)
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + 1e-4 * d, x[i] - 1e-4 * d
        g = f64(t.grad)
        assert abs((f(*up) - f(*down)) / 2e-4 - (g * d).sum()) <= 1e-4 * np.sqrt(((g * d) ** 2).sum() + 1), i


def test_head_norm_parts(dec):
    """One output used, frozen weights, no gradient at all, queries alone, a weight in another type and shape."""
    leaves, turn = head_case(dec, torch.float32, seed=30)
    q, k, wq, wk = leaves
    dec.head_norm(*leaves, *turn)[0].sum().backward()
    assert q.grad.any() and not k.grad.any() and not wk.grad.any()
    first = q.grad.clone()
    frozen = q.detach().requires_grad_()
    dec.head_norm(frozen, k.detach(), wq.detach(), wk.detach(), *turn)[0].sum().backward()
    assert torch.equal(frozen.grad, first)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        dec.head_norm(*(t.detach() for t in leaves), *turn)
    assert not any(t.dtype == torch.uint8 for t in kept)
    alone = q.detach().requires_grad_()
    y, none = dec.head_norm(alone, None, wq.detach(), None, *turn)
    y.sum().backward()
    assert none is None and torch.equal(alone.grad, first)
    b, w = q.detach().bfloat16().requires_grad_(), wq.detach().view(1, 1, 64).clone().requires_grad_()
    dec.head_norm(b, None, w, None, *turn)[0].float().sum().backward()
    assert w.grad.shape == (1, 1, 64) and w.grad.dtype == torch.float32 and b.grad.dtype == torch.bfloat16


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_gradients(dec, dtype):
    """Through a mean over rows, whose gradient is one number expanded, and through a sum of weighted rows."""
    s = randn((3, 10, 500), 40, 2.0, dtype).requires_grad_()
    index = torch.randint(-1, 500, (3, 10, 7), generator=torch.Generator().manual_seed(1)).cuda()
    teacher = randn((3, 10, 7), 41)
    loss = dec.distill_loss(s, index, teacher, 2.0)
    want, stats = dec.distill_forward(s.detach(), index, teacher, 2.0)
    assert torch.equal(loss, want)
    loss.mean().backward(retain_graph=True)
    gl = torch.full((3, 10), 1.0 / 30, device="cuda")
    assert torch.equal(s.grad, dec.distill_backward(gl, s.detach(), index, teacher, stats, 2.0))
    s.grad = None
    w = randn((3, 10), 42)
    (loss * w).sum().backward()
    assert torch.equal(s.grad, dec.distill_backward(w, s.detach(), index, teacher, stats, 2.0))


def test_distill_gradient_against_differences(dec):
    """As for the head norms: a hundred-term sum in fp32 against central differences in 64 bits."""
    s = randn((5, 300), 50, 2.0).requires_grad_()
    index = torch.randint(0, 300, (5, 9), generator=torch.Generator().manual_seed(2)).cuda()
    teacher, gl = randn((5, 9), 51), randn((5,), 52)
    (dec.distill_loss(s, index, teacher, 1.5) * gl).sum().backward()
    x, i, t, g = f64(s), index.cpu().numpy(), f64(teacher), f64(s.grad)
    d = np.random.default_rng(1).standard_normal(x.shape)
    f = lambda x: (ref.distill(x, i, t, 1.5) * f64(gl)).sum()
    assert abs((f(x + 1e-4 * d) - f(x - 1e-4 * d)) / 2e-4 - (g * d).sum()) <= 1e-4 * np.sqrt(((g * d) ** 2).sum() + 1)


# -- streams, graphs, far offsets -------------------------------------------------------------------------------------------


def every_operator(dec, x):
    """All calls, forward and backward, on the tensors of x."""
    y = dec.embed(x["tokens"], x["w"], 1.5)
    out = dec.head_norm_forward(x["q"], x["k"], x["wq"], x["wk"], x["cos"], x["sin"], x["positions"], fmt=1)
    g = dec.head_norm_backward(x["q"], x["k"], out[4], out[5], out[2], out[3], x["wq"], x["wk"], x["cos"], x["sin"], x["positions"])
    loss, stats = dec.distill_forward(x["s"], x["index"], x["teacher"])
    return [y, dec.embed_backward(x["tokens"], x["gy"], 200, 0.5), dec.embed_backward(x["many"], x["far"], 70000, 0.5), *out[:4], out[4].codes, out[5].scales, *g, loss, stats,
            dec.distill_backward(loss, x["s"], x["index"], x["teacher"], stats)]


def operands(dec, seed):
    g = torch.Generator().manual_seed(seed)
    cos, sin = dec.rotary_table(100, 64)
    ints = lambda hi, *shape: torch.randint(0, hi, shape, generator=g).cuda()
    return dict(tokens=ints(200, 3, 100), w=randn((200, 96), seed), gy=randn((3, 100, 96), seed + 1), many=ints(70000, 9000), far=randn((9000, 8), seed + 2),
                q=randn((3, 100, 4, 64), seed + 3), k=randn((3, 100, 2, 64), seed + 4), wq=randn((64,), seed + 5), wk=randn((64,), seed + 6), cos=cos, sin=sin,
                positions=ints(100, 3, 100), s=randn((20, 30000), seed + 7, 2.0), index=ints(30000, 20, 9), teacher=randn((20, 9), seed + 8))


def test_other_streams_and_graphs(dec):
    """The calls on another stream, and captured into two graphs that are replayed in turn on new inputs: the same bits as
    called one by one.  The workspaces of a graph are its own."""
    x = [operands(dec, 100), operands(dec, 200)]
    want = [every_operator(dec, t) for t in x]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = every_operator(dec, x[0])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graphs, outs = [], []
    for t in x:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(every_operator(dec, t))
    for turn in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o, t in zip(outs, x):
            assert all(torch.equal(a, b) for a, b in zip(o, every_operator(dec, t))), turn
        for k, t in enumerate(x):
            for name, v in operands(dec, 300 + 10 * turn + k).items():
                t[name].copy_(v)


def test_two_calls_at_once(dec):
    """The same operator on two streams at a time, each with its own workspace."""
    x = [operands(dec, 400), operands(dec, 500)]
    want = [every_operator(dec, t) for t in x]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = every_operator(dec, x[i])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_training_step_graph(dec):
    """Forward and backward through the differentiable forms, captured once and replayed: the gradients of an eager step on
    the same inputs.  The leaves are the step's own."""
    x = operands(dec, 600)
    head = randn((500, 256), 601, 0.1)

    def step():
        w, wq, wk, h = (t.detach().requires_grad_() for t in (x["w"], x["wq"], x["wk"], head))
        e = dec.embedding(x["tokens"], w, 2.0)[..., :64].unsqueeze(2)
        q, k = dec.head_norm(e * x["q"], e * x["k"], wq, wk, x["cos"], x["sin"], x["positions"])
        y = (q * k.repeat_interleave(2, 2)).flatten(2)
        loss = dec.distill_loss(y @ h.t(), x["index"].repeat(15, 1).view(3, 100, 9) % 500, x["teacher"].repeat(15, 1).view(3, 100, 9)).mean()
        return torch.autograd.grad(loss, (w, wq, wk, h))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (700, 800):
        for name, v in operands(dec, seed).items():
            x[name].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_offsets_past_32_bits(dec):
    """Tensors of more than 2^32 bytes and 2^31 elements: their last rows are those of a call on these alone."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 60 GB")
    bf16 = torch.bfloat16
    vocab, cols = 540000, 4096
    w = torch.zeros(vocab, cols, dtype=bf16, device="cuda")
    w[-3:] = randn((3, cols), 1, dtype=bf16)
    tokens = torch.tensor([vocab - 1, 0, vocab - 3, vocab - 1], device="cuda")
    assert torch.equal(dec.embed(tokens, w), w[tokens])
    gy = randn((4, cols), 2, dtype=bf16)
    small = dec.embed_backward(torch.tensor([2, 3, 0, 2], device="cuda"), gy, 4)   # the same order of sums
    del w
    gw = dec.embed_backward(tokens, gy, vocab)
    assert torch.equal(gw[-3:], small[:3]) and torch.equal(gw[0], small[3]) and not gw[1:-3].any()
    del gw
    rows, v = 17000, 128000
    s = torch.zeros(rows, v, dtype=bf16, device="cuda")
    s[-2:] = randn((2, v), 3, 2.0, bf16)
    index = torch.full((rows, 5), -1, device="cuda")
    index[-2:] = torch.randint(0, v, (2, 5), device="cuda")
    teacher = randn((rows, 5), 4)
    loss, stats = dec.distill_forward(s, index, teacher)
    gs = dec.distill_backward(loss, s, index, teacher, stats)
    # few rows are shared by several CTAs: sums in another order, so compared with the definition's bounds
    want = ref.distill(f64(s[-2:]), index[-2:].cpu().numpy(), f64(teacher[-2:]), 1.0)
    assert np.allclose(f64(loss[-2:]), want, rtol=1e-5) and not loss[:-2].any()
    assert torch.equal(gs[-2:], dec.distill_backward(loss[-2:], s[-2:], index[-2:], teacher[-2:], stats[-2:])) and not gs[:-2].any()
    del s, gs
    tokens_n = 270000
    cos, sin = dec.rotary_table(8, 128)
    q = torch.ones(1, tokens_n, 64, 128, dtype=bf16, device="cuda")
    q[:, -4:] = randn((1, 4, 64, 128), 5, dtype=bf16)
    at = torch.arange(tokens_n, device="cuda") % 8
    y, _, r, _, p, _ = dec.head_norm_forward(q, None, None, None, cos, sin, at, fmt=1)
    ys, _, rs, _, ps, _ = dec.head_norm_forward(q[:, -4:], None, None, None, cos, sin, at[-4:], fmt=1)
    assert torch.equal(y[:, -4:], ys) and torch.equal(p.codes[-256:], ps.codes) and torch.equal(r[:, -4:], rs)
    gx = dec.head_norm_backward(y, None, p, None, r, None, None, None, cos, sin, at)[0]
    assert torch.equal(gx[:, -4:], dec.head_norm_backward(ys, None, ps, None, rs, None, None, None, cos, sin, at[-4:])[0])


# -- a decoder ----------------------------------------------------------------------------------------------------------------


class Attention(torch.nn.Module):
    def __init__(self, dec, hooks, width, heads, kv, cols):
        super().__init__()
        self.heads, self.kv, self.cols = heads, kv, cols
        self.norm = torch.nn.RMSNorm(width, eps=1e-5)
        self.q, self.k, self.v = (torch.nn.Linear(width, n * cols, bias=False) for n in (heads, kv, kv))
        self.o = torch.nn.Linear(heads * cols, width, bias=False)
        self.head_norm = dec.HeadNorm(cols)
        self.qk, self.av = hooks.BatchedMatmul(), hooks.BatchedMatmul()

    def forward(self, x, cos, sin):
        h = self.norm(x)
        q, k = self.head_norm(self.q(h).unflatten(-1, (self.heads, self.cols)), self.k(h).unflatten(-1, (self.kv, self.cols)), cos, sin)
        v = self.v(h).unflatten(-1, (self.kv, self.cols))
        many = self.heads // self.kv
        q, k, v = q.transpose(1, 2), k.repeat_interleave(many, 2).transpose(1, 2), v.repeat_interleave(many, 2).transpose(1, 2)
        mask = torch.full((x.shape[1],) * 2, float("-inf"), device=x.device, dtype=x.dtype).triu(1)
        p = (self.qk(q, k.transpose(2, 3)) / self.cols ** 0.5 + mask).softmax(-1)
        return x + self.o(self.av(p, v).transpose(1, 2).flatten(2))


class Decoder(torch.nn.Module):
    def __init__(self, dec, hooks, vocab=301, width=64, layers=2):
        super().__init__()
        self.embed = dec.ScaledEmbedding(vocab, width, width ** 0.5, padding_idx=0)
        self.blocks = torch.nn.ModuleList([Attention(dec, hooks, width, 4, 2, 32) for _ in range(layers)])
        self.head = torch.nn.Linear(width, vocab, bias=False)
        self.turn = dec.rotary_table(64, 32)

    def forward(self, tokens):
        x = self.embed(tokens)
        for b in self.blocks:
            x = b(x, *(t.to(x.device) for t in self.turn))
        return self.head(x)


def plain_gradients(net, tokens, index, teacher):
    """The same model in 64 bits with torch's own operators; gradients by parameter name."""
    p = {n: t.detach().double().requires_grad_() for n, t in net.named_parameters()}
    x = torch.nn.functional.embedding(tokens, p["embed.weight"], padding_idx=0) * net.embed.scale

    def rms(x, w, eps=1e-5):
        return x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * w

    cos, sin = (t.double()[: tokens.shape[1], None, :] for t in net.turn)

    def turned(n):
        a, b = n.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    for i, b in enumerate(net.blocks):
        w = lambda name: p["blocks.%d.%s" % (i, name)]
        h = rms(x, w("norm.weight"))
        q, k, v = ((h @ w(n + ".weight").t()).unflatten(-1, (m, 32)) for n, m in (("q", 4), ("k", 2), ("v", 2)))
        q, k = turned(rms(q, w("head_norm.weight_q"))), turned(rms(k, w("head_norm.weight_k")))
        k, v = k.repeat_interleave(2, 2), v.repeat_interleave(2, 2)
        a = torch.einsum("bthc,bshc->bhts", q, k) / 32 ** 0.5
        a = a.masked_fill(torch.ones(a.shape[-2:], device=a.device, dtype=torch.bool).triu(1), float("-inf")).softmax(-1)
        x = x + torch.einsum("bhts,bshc->bthc", a, v).flatten(2) @ w("o.weight").t()
    log_q = (x @ p["head.weight"].t()).log_softmax(-1).gather(-1, index.clamp(min=0))
    log_p = teacher.double().masked_fill(index < 0, float("-inf")).log_softmax(-1)
    loss = torch.where(index >= 0, log_p.exp() * (log_p - log_q), 0.0).sum(-1).mean()
    names = [n for n, _ in net.named_parameters()]
    return float(loss.detach()), dict(zip(names, torch.autograd.grad(loss, [p[n] for n in names])))


@contextlib.contextmanager
def a_decoder(ampq, dec):
    from paper_2505_13060_b200 import hooks

    torch.manual_seed(3)
    net = Decoder(dec, hooks).cuda()
    ctx = ampq.Context(0, torch.cuda.current_stream().cuda_stream)
    ctx.set_formats([0, 1])
    tokens = torch.randint(1, 301, (2, 24), generator=torch.Generator().manual_seed(1)).cuda()
    tokens[1, 20:] = 0
    index = torch.randint(0, 301, (2, 24, 8), generator=torch.Generator().manual_seed(2)).cuda()
    index[1, 19:, 3:] = -1
    teacher = randn((2, 24, 8), 4)
    try:
        yield hooks, net, ctx, tokens, index, teacher
    finally:
        ctx.destroy()


def test_decoder_gradients(ampq, dec):
    """Embedding, norms, head norms, products, loss: one pass in fp32 against the same model in 64 bits.  Some thirty
    operations in a row with sums of at most 301 terms each lose 30 * 301 * 2^-24 = 6e-4 of a gradient's norm at the very
    worst; rounding errors of either sign add up to their root, 3e-5: the bound is between the two."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        loss = dec.distill_loss(net(tokens), index, teacher).mean()
        loss.backward()
        want, grads = plain_gradients(net, tokens, index, teacher)
        assert abs(float(loss.detach()) - want) <= 2e-4 * abs(want)
        for n, t in net.named_parameters():
            assert float((t.grad.double() - grads[n]).norm()) <= 2e-4 * float(grads[n].norm()), n
        assert not net.embed.weight.grad[0].any()


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_decoder_calibration(ampq, dec, fmt):
    """A calibration of the decoder with the loss from the teacher's lists: every layer is scored, twice the same, and with
    checkpoints the head norms keep no input in full."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        results, kept = [], []
        for _ in range(2):
            cal = hooks.Calibrator(ctx, net, 2, checkpoint=fmt)
            cal.begin()
            for r in range(2):
                kept.clear()
                seen = []
                handle = net.blocks[0].head_norm.register_forward_pre_hook(lambda m, args: seen.extend(args[:2]))   # held: their memory is not used again
                net.zero_grad()
                with cal.sample(r), torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.data_ptr()) or t, lambda t: t):
                    dec.distill_loss(net(tokens[r:r + 1]), index[r:r + 1], teacher[r:r + 1]).mean().backward()
                handle.remove()
                assert len(seen) == 2 and any(a.data_ptr() in kept for a in seen) == (fmt == 0)
            results.append(cal.end())
            assert len(results[-1]) == 2 * 6 + 1
            assert all(len(f["s_per_sample"]) == 2 and (f["s_per_sample"] > 0).all() for f in results[-1])
        grads = [t.grad for t in net.parameters()]
        assert all(g is not None and bool(g.isfinite().all()) for g in grads)
        for a, b in zip(*results):
            assert np.array_equal(a["s_per_sample"], b["s_per_sample"])


def test_divergence_of_a_configuration(ampq, dec):
    """The divergence of a quantised model from its own logits: that of a list of the model itself where nothing is
    quantised, larger where everything is, and the model is left as it was."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        cal = hooks.Calibrator(ctx, net, 1)
        forward = lambda: net(tokens)
        logits = forward().detach()
        before = [t.detach().clone() for t in net.parameters()]
        none = cal.divergence(forward, [0] * 13, top=301)
        full = cal.divergence(forward, [1] * 13, top=301)
        assert none.shape == (2, 24) and none.dtype == torch.float32
        # the divergence of a row from all of itself is 0: what is left is the rounding of sums of 301 terms
        assert float(none.abs().max()) <= 301 * 8 * U
        assert float(full.min()) > float(none.abs().max())
        with cal.quantised([1] * 13):
            got = forward().detach()
        # and that of all columns is the divergence of two softmaxes: in 64 bits of the same logits
        p, q = logits.double().log_softmax(-1), got.double().log_softmax(-1)
        want = (p.exp() * (p - q)).sum(-1)
        assert float((full.double() - want).abs().max()) <= 301 * 16 * U
        assert all(torch.equal(a, b) for a, b in zip(before, net.parameters()))
        cal.begin()   # the calibrator is ready for a pass
        with cal.sample(0):
            net(tokens[:1]).square().mean().backward()
        assert len(cal.end()) == 13


def test_head_norm_module_in_a_calibration(ampq, dec):
    """Outside of samples, and without gradients inside of one, the module keeps what it is told to; a format that the call
    names is not replaced; the forward pass is the same one."""
    with a_decoder(ampq, dec) as (hooks, net, ctx, tokens, index, teacher):
        m = net.blocks[0].head_norm
        cos, sin = (t.cuda() for t in net.turn)
        q, k = randn((1, 24, 4, 32), 1).requires_grad_(), randn((1, 24, 2, 32), 2)
        want = m(q, k, cos, sin)
        cal = hooks.Calibrator(ctx, net, 1, checkpoint=1)
        cal.begin()

        def codes(**fmt):
            kept = []
            with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
                y = m(q, k=k, cos=cos, sin=sin, positions=None, **fmt)
            assert all(torch.equal(a, b) for a, b in zip(y, want))
            return [t for t in kept if t.dtype == torch.uint8]

        assert not codes()
        with cal.sample(0):
            by_default, e5m2 = codes(), codes(fmt=2)
            with torch.no_grad():
                assert not codes()
            net(tokens[:1]).square().mean().backward()
        assert len(by_default) == 4 and not torch.equal(by_default[0], e5m2[0])
        assert not codes() and len(codes(fmt=2)) == 4
        cal.end()
