"""Embedding, head norms with rotation and distillation on the GPU, against their
definitions in 64 bits on the host.

Bounds: U = 2^-24 is half a step of fp32, H half a step of the output's type.  An fp32
sum of n terms, in any order, is off by at most n U of the sum of their absolute values.
"""
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


@pytest.fixture(scope="module")
def ckpt(ampq):
    from paper_2505_13060_b200 import checkpoint

    return checkpoint


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, tol, what=""):
    off = np.abs(f64(got) - want)
    assert off.shape == np.broadcast_shapes(want.shape, np.shape(tol)), (what, got.shape)
    assert (off <= tol).all(), (what, (off / np.maximum(tol, 1e-300)).max())


def randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


# -- embedding ---------------------------------------------------------------------------------------------------------


def check_embed(dec, tokens, w, scale, index=torch.int64):
    y = dec.embed(tokens.to(index), w, scale)
    s = float(np.float32(scale))
    want = f64(w)[tokens.cpu().numpy()] * s
    assert y.dtype == w.dtype and y.shape == (*tokens.shape, w.shape[1])
    # one product rounded in fp32, then to the type
    h = HALF_STEP[w.dtype]
    within(y, want, (U + h * (1 + U) if h > U else U) * np.abs(want))


def check_embed_grad(dec, tokens, gy, vocab, scale, padding=None, index=torch.int64):
    gw = dec.embed_backward(tokens.to(index), gy, vocab, scale, padding)
    want, size, count = ref.embed_grad(tokens.reshape(-1).cpu().numpy(), f64(gy).reshape(-1, gy.shape[-1]), vocab, float(np.float32(scale)), padding)
    assert gw.dtype == gy.dtype and gw.shape == (vocab, gy.shape[-1])
    within(gw, want, (count[:, None] + 2) * U * size * (1 + 2.0 ** -8) + HALF_STEP[gy.dtype] * np.abs(want))
    return gw


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_embed_sizes(dec, dtype, index):
    g = torch.Generator().manual_seed(3)
    for n, vocab, cols in [(1, 1, 1), (1, 9, 4096), (3, 5, 33), (8, 1000, 257), (70, 70, 8), (300, 11, 16), (513, 4001, 130), (2049, 300, 24), (5, 40, 9000),
                           (4100, 70000, 3)]:
        tokens = torch.randint(0, vocab, (n,), generator=g).cuda()
        check_embed(dec, tokens, randn((vocab, cols), dtype, n), 1.7, index)
        gy = randn((n, cols), dtype, n + 1)
        check_embed_grad(dec, tokens, gy, vocab, 0.3, None, index)
        check_embed_grad(dec, tokens, gy, vocab, 1.0, int(tokens[0]), index)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_embed_layouts(dec, dtype):
    """Tables and gradients inside wider ones, rows that start anywhere, batches, expanded gradients, tokens that are a slice."""
    tokens = torch.randint(0, 50, (3, 14), generator=torch.Generator().manual_seed(0)).cuda()
    for extra, at in ((16, 0), (3, 1)):
        w = randn((50, 72 + extra), dtype, 1)[:, at:at + 72]
        check_embed(dec, tokens[:, ::2], w, 1.0)
        check_embed_grad(dec, tokens[:, ::2], randn((3, 7, 72 + extra), dtype, 2)[..., at:at + 72], 50, 2.0)
    check_embed(dec, tokens, randn((72, 50), dtype, 3).t(), 1.0)
    check_embed_grad(dec, tokens, randn((1, 1, 72), dtype, 4).expand(3, 14, 72), 50, 1.0)
    check_embed_grad(dec, tokens, randn((3, 72, 14), dtype, 4).transpose(1, 2), 50, 1.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_embed_grad_runs(dec, dtype):
    """Runs of equal tokens of every length around the pieces that they are cut into, one token for all, all different."""
    vocab, cols = 400, 40
    lengths = [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 700]
    tokens = torch.cat([torch.full((m,), 3 * i) for i, m in enumerate(lengths)])
    order = torch.randperm(len(tokens), generator=torch.Generator().manual_seed(1))
    for t in (tokens, tokens[order], torch.full((3000,), 399), torch.zeros(2048, dtype=torch.int64), torch.arange(400), torch.arange(399, -1, -1)):
        check_embed_grad(dec, t.cuda(), randn((len(t), cols), dtype, 5), vocab, 1.0)


def test_embed_grad_many_tokens(dec):
    """Enough tokens for the longest pieces and several tiles of the sort, most of them one padding token that counts."""
    g = torch.Generator().manual_seed(2)
    tokens = torch.randint(0, 70000, (50000,), generator=g)
    tokens[torch.rand(50000, generator=g) < 0.6] = 65537
    check_embed_grad(dec, tokens.cuda(), randn((50000, 8), torch.float32, 6), 70000, 1.0)
    check_embed_grad(dec, tokens.cuda(), randn((50000, 8), torch.bfloat16, 7), 70000, 1.0, 65537)


def test_embed_repeats_itself(dec):
    tokens = torch.randint(0, 37, (5000,), generator=torch.Generator().manual_seed(4)).cuda()
    gy = randn((5000, 300), torch.float32, 8)
    first = dec.embed_backward(tokens, gy, 37)
    for _ in range(5):
        assert torch.equal(dec.embed_backward(tokens, gy, 37), first)


def test_embed_nothing(dec):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert dec.embed(none, randn((4, 8), torch.float32, 0)).shape == (0, 8)
    assert dec.embed(torch.zeros(3, dtype=torch.int64, device="cuda"), torch.empty(4, 0, device="cuda")).shape == (3, 0)
    gw = dec.embed_backward(none, torch.empty(0, 8, device="cuda"), 5)
    assert torch.equal(gw, torch.zeros(5, 8, device="cuda"))
    assert dec.embed_backward(none, torch.empty(0, 8, device="cuda"), 0).shape == (0, 8)
    assert dec.embed_backward(torch.zeros(3, dtype=torch.int64, device="cuda"), torch.empty(3, 0, device="cuda"), 5).shape == (5, 0)


def test_embed_outside_the_table(dec):
    """Tokens that are no row: NaN forward, no part in any gradient.  Inf and NaN stay in their own rows."""
    tokens = torch.tensor([0, -1, 4, 5, 2 ** 40, 4, -2 ** 40], device="cuda")
    w = randn((5, 24), torch.float32, 1)
    y = dec.embed(tokens, w, 2.0)
    bad = torch.tensor([False, True, False, True, True, False, True])
    assert bool(y[bad.cuda()].isnan().all()) and torch.equal(y[~bad.cuda()], w[tokens[~bad.cuda()]] * 2.0)
    gy = randn((7, 24), torch.float32, 2)
    gy[0, 3], gy[2, 5] = float("inf"), float("nan")
    gw = dec.embed_backward(tokens, gy, 5)
    assert bool((gw[1:4] == 0).all()) and float(gw[0, 3]) == float("inf") and bool(gw[4, 5].isnan())
    assert int(gw.isfinite().sum()) == 5 * 24 - 2
    small = tokens.clamp(-2, 6).int()
    assert torch.equal(dec.embed_backward(small, gy, 5).nan_to_num(), gw.nan_to_num())


def test_embed_grad_writes_its_rows_only(ampq, dec):
    tokens, gy = torch.tensor([1, 1, 3], device="cuda"), randn((3, 33), torch.bfloat16, 1)
    full = torch.full((7, 33), 5.0, dtype=torch.bfloat16, device="cuda")
    need = dec._embed_backward_bytes(0, ampq.BF16, 3, 4, 33)
    ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    rc = ampq.lib().ampq_embed_backward(0, st, ampq.BF16, ampq.I64, tokens.data_ptr(), 3, gy.data_ptr(), 33, 4, 33, 1.0, -1, full.data_ptr(), ws.data_ptr(), need)
    assert rc == 0 and torch.equal(full[:4], dec.embed_backward(tokens, gy, 4))
    assert bool((full[4:] == 5.0).all()) and bool((ws[need:] == 0xA5).all())
    assert ampq.lib().ampq_embed_backward(0, st, ampq.BF16, ampq.I64, tokens.data_ptr(), 3, gy.data_ptr(), 33, 4, 33, 1.0, -1, full.data_ptr(), ws.data_ptr(),
                                          need - 1) == ampq.ERR_INVALID


# -- norms of heads ------------------------------------------------------------------------------------------------------


def laid(t, layout):
    """The same values [batch, tokens, heads, cols]: contiguous, part of a wider row, heads before tokens, or at an odd place."""
    if layout == "plain":
        return t
    b, n, h, c = t.shape
    if layout == "fused":
        full = torch.full((b, n, h + 2, c), 9.0, dtype=t.dtype, device=t.device)
        out = full[:, :, 1:h + 1]
    elif layout == "heads first":
        out = torch.empty(b, h, n, c, dtype=t.dtype, device=t.device).transpose(1, 2)
    else:
        out = torch.full((b * n * h * (c + 1) + 1,), 9.0, dtype=t.dtype, device=t.device)[1:].view(b, n, h, c + 1)[..., :c]
    return out.copy_(t)


class HeadCase:
    def __init__(self, dec, dtype, batch, tokens, hq, hk, cols, rot, interleaved=False, layout="plain", own_positions=True, index=torch.int64, weights=None,
                 seed=0, fmt=0):
        self.__dict__.update(dtype=dtype, rot=rot, interleaved=interleaved, cols=cols, fmt=fmt)
        self.cos, self.sin = dec.rotary_table(200, rot)
        g = torch.Generator().manual_seed(seed)
        shape = (batch, tokens) if own_positions else (tokens,)
        self.positions = torch.randint(0, 200, shape, generator=g).to(index).cuda()
        wtype = weights or dtype
        self.q, self.k = (laid(randn((batch, tokens, h, cols), dtype, seed + h + i, 2.0), layout) for i, h in ((1, hq), (2, hk)))
        self.wq, self.wk = (None if weights == "none" else (1 + randn((cols,), torch.float32, seed + i, 0.3)).to(wtype) for i in (8, 9))
        self.gq, self.gk = (laid(randn((batch, tokens, h, cols), dtype, seed + h + i, 0.1), layout) for i, h in ((3, hq), (4, hk)))
        at = self.positions.long().cpu().numpy()
        self.c, self.s = (np.broadcast_to(f64(t)[at], (batch, tokens, rot // 2)) for t in (self.cos, self.sin))

    def angles(self):
        return self.cos, self.sin, self.positions

    def parts(self):
        ones = np.ones(self.cols)
        return (("q", self.q, self.gq, f64(self.wq) if self.wq is not None else ones), ("k", self.k, self.gk, f64(self.wk) if self.wk is not None else ones))


def check_heads(dec, c, backward=True):
    h, n, cols = HALF_STEP[c.dtype], c.rot, c.cols
    yq, yk, rq, rk, pq, pk = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles(), 1e-5, c.interleaved, c.fmt)
    for (name, x, _, w), y, r, p in zip(c.parts(), (yq, yk), (rq, rk), (pq, pk)):
        x = f64(x)
        want, size, rstd = ref.head_norm(x, w, c.c, c.s, n, 1e-5, c.interleaved)
        assert y.dtype == c.dtype and y.shape == x.shape and r.shape == x.shape[:3]
        # the sum of cols squares (each rounded too), the mean, eps, half of that through the root, the root and its reciprocal
        e = (cols / 2 + 4) * U
        within(r, rstd, e * rstd, name + " rstd")
        # two products, and in the turned columns one more and an addition; then the type
        within(y, want, (e + 5 * U) * size * (1 + h) + h * np.abs(want), name + " y")
        if c.fmt:
            codes, scales = kept_ref.pack(x.reshape(-1, cols), c.fmt)
            assert np.array_equal(p.scales.cpu().numpy(), scales) and np.array_equal(p.codes.cpu().numpy(), codes), name
        else:
            assert p is None
    if not backward:
        return
    xq, xk = (pq, pk) if c.fmt else (c.q, c.k)
    gxq, gxk, gwq, gwk = dec.head_norm_backward(c.gq, c.gk, xq, xk, rq, rk, c.wq, c.wk, *c.angles(), c.interleaved)
    for (name, x, gy, w), r, p, gx, gw in zip(c.parts(), (rq, rk), (pq, pk), (gxq, gxk), (gwq, gwk)):
        v = f64(x) if not c.fmt else kept_ref.unpack(p.codes.cpu().numpy(), p.scales.cpu().numpy(), cols, c.fmt).reshape(x.shape)
        want, want_w, u, mean, gsize = ref.head_norm_grad(f64(gy), v, f64(r), w, c.c, c.s, n, c.interleaved)
        # u has four roundings; the mean cols + 7 and the product with h two more; then the difference, rstd and the type
        tol = f64(r)[..., None] * U * (7 * u + (cols + 12) * mean) * (1 + h) + h * np.abs(want)
        within(gx, want, tol, name + " gx")
        if gw is not None:
            rows = gy.shape[0] * gy.shape[1] * gy.shape[2]
            hw = HALF_STEP[gw.dtype]
            within(gw, want_w, (rows + 6) * U * gsize * (1 + hw) + hw * np.abs(want_w), name + " gw")
        else:
            assert w.min() == w.max() == 1.0


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_heads_sizes(dec, dtype, interleaved, fmt):
    for cols, rot in [(2, 0), (2, 2), (6, 4), (16, 16), (32, 32), (34, 16), (48, 32), (64, 64), (64, 32), (72, 36), (80, 80), (80, 40), (96, 96), (100, 50),
                      (128, 128), (128, 64), (128, 0), (160, 160), (192, 64), (254, 254), (256, 256), (256, 128)]:
        for batch, tokens, hq, hk in [(2, 3, 3, 1), (1, 1, 9, 9)]:
            check_heads(dec, HeadCase(dec, dtype, batch, tokens, hq, hk, cols, rot, interleaved, seed=cols, fmt=fmt))


@pytest.mark.parametrize("layout", ["plain", "fused", "heads first", "odd"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_heads_layouts(dec, dtype, layout):
    for cols, rot, interleaved, fmt in [(64, 64, False, 0), (128, 64, True, 1), (40, 20, False, 2)]:
        check_heads(dec, HeadCase(dec, dtype, 3, 17, 5, 2, cols, rot, interleaved, layout, seed=1, fmt=fmt))


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_heads_of_many_tokens(dec, dtype, fmt):
    """More runs of heads than a grid has warps, in both passes."""
    check_heads(dec, HeadCase(dec, dtype, 2, 700, 16, 4, 64, 64, seed=2, fmt=fmt))
    check_heads(dec, HeadCase(dec, dtype, 1, 3001, 1, 1, 128, 128, True, "fused", seed=3, fmt=fmt))


def test_heads_weights_and_positions(dec):
    for weights in ("none", torch.float32, torch.bfloat16):
        for own, index in ((True, torch.int32), (False, torch.int64)):
            check_heads(dec, HeadCase(dec, torch.bfloat16, 2, 9, 4, 2, 64, 32, own_positions=own, index=index, weights=weights, seed=5))
    c = HeadCase(dec, torch.float32, 2, 9, 4, 2, 64, 32, seed=6)
    rows = torch.arange(9, device="cuda")
    same = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, c.cos, c.sin, rows)
    for a, b in zip(dec.head_norm_forward(c.q, c.k, c.wq, c.wk, c.cos, c.sin)[:4], same):   # no positions: the token's place
        assert torch.equal(a, b)
    wide = torch.zeros(2, 18, dtype=torch.int64, device="cuda")
    wide[:, ::2] = c.positions
    for a, b in zip(dec.head_norm_forward(c.q, c.k, c.wq, c.wk, c.cos, c.sin, wide[:, ::2])[:2],
                    dec.head_norm_forward(c.q, c.k, c.wq, c.wk, c.cos, c.sin, c.positions)):
        assert torch.equal(a, b)
    # no rotation, and weights for the keys alone
    y, _, r = dec.head_norm_forward(c.q, c.k, None, c.wk)[:3]
    want, size, rstd = ref.head_norm(f64(c.q), np.ones(64), np.zeros((2, 9, 0)), np.zeros((2, 9, 0)), 0, 1e-5, False)
    within(y, want, (32 + 4 + 5) * U * size + U * np.abs(want))
    assert [t is None for t in dec.head_norm_backward(c.gq, c.gk, c.q, c.k, r, dec.head_norm_forward(c.k, None)[2], None, c.wk)] == [False, False, True, False]


def test_queries_alone_and_other_dimensions(dec):
    """Keys may be left out, and the tensors may have fewer or more leading dimensions."""
    c = HeadCase(dec, torch.float32, 4, 6, 3, 2, 32, 32, seed=7)
    yq, yk, rq, rk, _, _ = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles())
    alone = dec.head_norm_forward(c.q, None, c.wq, None, *c.angles())
    assert torch.equal(alone[0], yq) and alone[1] is None and torch.equal(alone[2], rq) and alone[3] is None
    five = dec.head_norm_forward(c.q.view(2, 2, 6, 3, 32), c.k.view(2, 2, 6, 2, 32), c.wq, c.wk, c.cos, c.sin, c.positions.view(2, 2, 6))
    assert torch.equal(five[0].view_as(yq), yq) and torch.equal(five[1].view_as(yk), yk) and five[2].shape == (2, 2, 6, 3)
    three = dec.head_norm_forward(c.q[1], c.k[1], c.wq, c.wk, c.cos, c.sin, c.positions[1])
    assert torch.equal(three[0], yq[1]) and torch.equal(three[3], rk[1])
    g = dec.head_norm_backward(c.gq, c.gk, c.q, c.k, rq, rk, c.wq, c.wk, *c.angles())
    a = dec.head_norm_backward(c.gq, None, c.q, None, rq, None, c.wq, None, *c.angles())
    assert torch.equal(a[0], g[0]) and a[1] is a[3] is None
    # The weight's gradient is a sum of 72 products whose order goes by the sizes, the keys' heads among them: each of the two is
    # off by at most (72 + 6) U of the absolute sum, as in check_heads, so they differ by twice that.
    size = ref.head_norm_grad(f64(c.gq), f64(c.q), f64(rq), f64(c.wq), c.c, c.s, 32, False)[4]
    within(a[2], f64(g[2]), 2 * 78 * U * size)


def test_heads_nothing(dec):
    for b, n, h, c in [(0, 3, 2, 8), (2, 0, 2, 8), (2, 3, 0, 8), (2, 3, 2, 0)]:
        q, k = torch.ones(b, n, h, c, device="cuda"), torch.ones(b, n, 1, c, device="cuda")
        w = torch.ones(c, device="cuda")
        yq, yk, rq, rk, pq, pk = dec.head_norm_forward(q, k, w, w, fmt=1)
        assert yq.shape == q.shape and yk.shape == k.shape and pq.rows == b * n * h
        g = dec.head_norm_backward(yq, yk, pq, pk, rq, rk, w, w)
        assert g[0].shape == q.shape and g[2].shape == (c,) and (b * n * h > 0 or not g[2].any())
        if c == 0:
            assert bool(rq.isnan().all()) and bool(rk.isnan().all())


def test_heads_not_finite(dec, ckpt):
    """An Inf or a NaN stays in its own head; a position without angles spoils the turned columns of its token alone."""
    c = HeadCase(dec, torch.float32, 1, 4, 3, 1, 64, 32, seed=8, fmt=1)
    c.q[0, 1, 2, 40], c.q[0, 2, 0, 3] = float("inf"), float("nan")
    yq, yk, rq, _, pq, _ = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles(), fmt=1)
    bad = ~yq.isfinite().all(3)
    assert bad[0].nonzero().tolist() == [[1, 2], [2, 0]] and float(rq[0, 1, 2]) == 0.0 and bool(rq[0, 2, 0].isnan())
    scales = pq.scales.view(4, 3, 2)
    assert (scales == 255).nonzero().tolist() == [[1, 2, 1], [2, 0, 0]]
    c = HeadCase(dec, torch.float32, 1, 4, 3, 1, 64, 32, seed=8)
    good = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles())
    for out in (200, -1, 2 ** 40):
        at = c.positions.clone()
        at[0, 2] = out
        y = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, c.cos, c.sin, at)
        assert bool(y[0][0, 2, :, :32].isnan().all()) and torch.equal(y[0][0, 2, :, 32:], good[0][0, 2, :, 32:])
        assert torch.equal(y[0][0, [0, 1, 3]], good[0][0, [0, 1, 3]])
        g = dec.head_norm_backward(c.gq, c.gk, c.q, c.k, good[2], good[3], c.wq, c.wk, c.cos, c.sin, at)
        assert bool(g[0][0, 2].isnan().all()) and bool(g[0][0, [0, 1, 3]].isfinite().all())


def test_heads_write_their_outputs_only(ampq, dec):
    """Strided outputs inside a larger tensor; what lies between the heads stays."""
    c = HeadCase(dec, torch.bfloat16, 2, 5, 3, 2, 64, 64, seed=9)
    want = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles())
    full = torch.full((2, 5, 8, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    sides = []
    for t, w, at, r in ((c.q, c.wq, 0, want[2]), (c.k, c.wk, 4, want[3])):
        s = dec._side(full[:, :, at:at + t.shape[2], :64], torch.empty_like(r), w, x=t)
        sides.append(s)
    st = torch.cuda.current_stream().cuda_stream
    rc = ampq.lib().ampq_head_norm_forward(0, st, ampq.BF16, ampq.BF16, ampq.I64, 0, 0, 2, 5, 64, 64, c.cos.data_ptr(), c.sin.data_ptr(), 200,
                                           c.positions.data_ptr(), 5, 1e-5, *sides)
    assert rc == 0
    assert torch.equal(full[:, :, :3, :64], want[0]) and torch.equal(full[:, :, 4:6, :64], want[1])
    full[:, :, :3, :64] = full[:, :, 4:6, :64] = 5.0
    assert bool((full == 5.0).all())


def test_heads_repeat_themselves(dec):
    c = HeadCase(dec, torch.bfloat16, 2, 500, 8, 2, 128, 128, seed=10, fmt=1)
    out = dec.head_norm_forward(c.q, c.k, c.wq, c.wk, *c.angles(), fmt=1)
    first = dec.head_norm_backward(c.gq, c.gk, out[4], out[5], out[2], out[3], c.wq, c.wk, *c.angles())
    for _ in range(5):
        again = dec.head_norm_backward(c.gq, c.gk, out[4], out[5], out[2], out[3], c.wq, c.wk, *c.angles())
        assert all(torch.equal(a, b) for a, b in zip(first, again))


# -- distillation ----------------------------------------------------------------------------------------------------------


def lists(rows, cols, top, seed, ragged=True):
    """Columns in any order, some of them twice; short lists, an entry missing here and there, rows without any."""
    g = torch.Generator().manual_seed(seed)
    index = torch.randint(0, cols, (rows, top), generator=g)
    if ragged:
        index[torch.rand(rows, top, generator=g) < 0.2] = -1
        index[2::5] = -7
    return index.cuda()


def check_distill(dec, s, index, teacher, T):
    rows, cols = s.shape
    loss, stats = dec.distill_forward(s, index, teacher, T)
    x, i, t = f64(s), index.cpu().numpy(), f64(teacher)
    used = (i >= 0).any(1)
    assert loss.dtype == torch.float32 and not loss[~torch.tensor(used).cuda()].any() and not stats[~torch.tensor(used).cuda()].any()
    m = x.max(1)
    with np.errstate(invalid="ignore"):
        d = np.where(np.isfinite(x), (m[:, None] - x) / T, 0.0)
        e = np.where(np.isfinite(x), np.exp(-d), 0.0)
    total = e.sum(1)
    assert np.array_equal(f64(stats)[used, 0], m[used])
    # A term: its difference, two products (3 U of the exponent) and an exponential (4 U), once for the term and once for each
    # time that it is put under a larger maximum, at most 48 times for vectors of a thread and merges of threads: the
    # exponents of these add up to the term's own.  Then additions: cols / 256 in a thread, 40 between threads.
    e_total = U * (cols / 256 + 40 + 4 * 49 + 6 * (e * d).sum(1) / total)
    within(stats[:, 1], np.where(used, total, 0.0), np.where(used, e_total * total, 0.0), "total")
    p, want = ref.targets(i, t, T), ref.distill(np.where(np.isfinite(x), x, -1e30), i, t, T)
    big = np.where(i >= 0, t, -np.inf).max(1, initial=-np.inf)
    with np.errstate(invalid="ignore"):
        a = np.where(i >= 0, np.abs(t - big[:, None]) / T, 0.0)
        listed = np.take_along_axis(x, np.maximum(i, 0), 1)
        b = np.where((i >= 0) & np.isfinite(listed), np.abs(listed - m[:, None]) / T, 0.0)
    e_list = U * (i.shape[1] + 12 + 6 * a.max(1, initial=0.0))
    logs = np.abs(np.log(total)) + np.abs(np.log(np.maximum(np.exp(-a).sum(1), 1)))
    tol = T * T * (e_total + e_list * (1 + (p * (a + b)).sum(1)) + 4 * U * (logs + (p * (a + b)).sum(1))) + 4 * U * np.abs(want)
    within(loss, want, np.where(used, tol, 0.0), "loss")

    gl = randn((rows,), torch.float32, rows)
    gs = dec.distill_backward(gl, s, index, teacher, stats, T)
    want, q, target = ref.distill_grad(f64(gl), np.where(np.isfinite(x), x, -1e30), i, t, T)
    h = HALF_STEP[s.dtype]
    assert gs.dtype == s.dtype and gs.shape == s.shape and not gs[~torch.tensor(used).cuda()].any()
    # q: exponent 3 U, exponential 4, the total's own error and its reciprocal, three products; p as above; a difference.
    # Below the smallest normal numbers (2^-126) results may be 0, and steps are 2^-133 in bf16.
    tol = np.abs(f64(gl))[:, None] * T * (q * (U * (3 * d + 9) + e_total[:, None]) + target * e_list[:, None] + 3 * U * (q + target) + 2.0 ** -125)
    within(gs, want, np.where(used[:, None], tol * (1 + h) + h * np.abs(want) + 2.0 ** -125, 0.0), "gs")


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_sizes(dec, dtype, index):
    for rows, cols, top, T in [(1, 1, 1, 1.0), (5, 2, 3, 1.0), (7, 31, 5, 2.0), (3, 33, 40, 0.5), (9, 1009, 8, 1.0), (2, 40000, 64, 1.0), (300, 257, 16, 4.0),
                               (1, 100003, 256, 1.0), (6, 8191, 1024, 1.5), (4, 70001, 1, 0.8)]:
        s = randn((rows, cols), dtype, cols, 2.5)
        teacher = randn((rows, top), torch.bfloat16 if top % 2 else torch.float32, top, 2.0)
        check_distill(dec, s, lists(rows, cols, top, rows).to(index), teacher, T)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_of_the_teacher_itself(dec, dtype):
    """Small divergences: what is left is what the list leaves out."""
    s = randn((40, 5000), dtype, 1, 3.0)
    value, index = s.topk(200, 1)
    check_distill(dec, s, index, value, 1.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_layouts(dec, dtype):
    """Logits, lists and gradients inside wider rows, rows that start anywhere, batches."""
    for extra, at in ((16, 0), (3, 1), (9, 5)):
        s = randn((23, 700 + extra), dtype, 2, 2.0)[:, at:at + 700]
        index, teacher = lists(23, 700, 20, 3)[:, ::2], randn((23, 13), torch.float32, 4)[:, 3:]
        check_distill(dec, s, index, teacher, 1.0)
    s, index, teacher = randn((2, 5, 90), dtype, 5), lists(10, 90, 4, 6).view(2, 5, 4), randn((2, 5, 4), torch.float32, 7)
    loss, stats = dec.distill_forward(s, index, teacher)
    flat, fstats = dec.distill_forward(s.view(10, 90), index.view(10, 4), teacher.view(10, 4))
    assert torch.equal(loss.view(10), flat) and torch.equal(stats.view(10, 2), fstats)
    one = torch.full((), 0.25, device="cuda").expand(2, 5)   # the gradient of a mean is one number expanded
    gs = dec.distill_backward(one, s, index, teacher, stats)
    assert torch.equal(gs, dec.distill_backward(one.contiguous(), s, index, teacher, stats)) and gs.shape == s.shape
    gl = randn((5, 2), torch.float32, 8).t()
    assert torch.equal(dec.distill_backward(gl, s, index, teacher, stats), dec.distill_backward(gl.contiguous(), s, index, teacher, stats))


@pytest.mark.parametrize("low", [float("-inf"), "lowest"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_masked_columns(dec, dtype, low):
    """Masked columns of -Inf or of the type's lowest value have no part; a row of nothing but the lowest value is uniform."""
    value = torch.finfo(dtype).min if low == "lowest" else low
    s = randn((12, 3001), dtype, 9, 2.0)
    s[:, 2900:] = value
    s[:, 100:1300] = value
    s[4, :2899] = value
    index = torch.randint(1300, 2900, (12, 6), generator=torch.Generator().manual_seed(2)).cuda()
    index[4] = 2899
    check_distill(dec, s, index, randn((12, 6), torch.float32, 10), 1.0)
    if low == "lowest":
        flat = torch.full((2, 500), value, dtype=dtype, device="cuda")
        teacher = randn((2, 6), torch.float32, 11) * 0
        loss, stats = dec.distill_forward(flat, index[:2] - 1290, teacher)
        # these lists name columns behind the 500th, which are none
        assert bool((stats[:, 1] == 500).all()) and (index[:2] - 1290).amax(1).gt(499).all() and bool(loss.isnan().all())
        loss, stats = dec.distill_forward(flat, (index[:2] - 1290) % 500, teacher)
        assert bool((stats[:, 1] == 500).all()) and np.allclose(f64(loss), [np.log(500) - np.log(6)] * 2, rtol=1e-6)


def test_distill_not_finite(dec):
    """Where the definition has no number there is NaN (or +Inf), in that row alone; rows without entries are not read."""
    s = randn((9, 400), torch.float32, 12, 2.0)
    index, teacher = lists(9, 400, 5, 13, ragged=False), randn((9, 5), torch.float32, 14)
    s[0, 17], s[1, 3], s[2, :] = float("nan"), float("inf"), float("-inf")
    s[3, :] = float("nan")
    index[3] = -1
    s[4, index[4, 0]] = float("-inf")          # the teacher gives it a probability
    s[5, index[5, 0]] = float("-inf")
    teacher[5, index[5] == index[5, 0]] = float("-inf")   # the teacher gives it none
    index[6, 2] = 400                           # no column
    teacher[7, :] = float("-inf")
    loss, stats = dec.distill_forward(s, index, teacher)
    want = [True, True, True, False, False, False, True, True, False]
    assert loss.isnan().tolist() == want and float(loss[3]) == 0.0 and float(loss[4]) == float("inf") and bool(loss[5].isfinite())
    gs = dec.distill_backward(torch.ones(9, device="cuda"), s, index, teacher, stats)
    assert bool(gs[0].isnan().all()) and not gs[3].any() and bool(gs[4].isfinite().all()) and bool(gs[5].isfinite().all()) and bool(gs[8].isfinite().all())
    assert bool(gs[6, index[6][index[6] < 400]].isnan().all()) and bool(gs[7, index[7]].isnan().all())
    assert abs(float(gs[4].double().sum())) < 1e-5 and abs(float(gs[5].double().sum())) < 1e-5


def test_distill_nothing(dec):
    none = torch.empty(0, 3, dtype=torch.int64, device="cuda")
    loss, stats = dec.distill_forward(torch.empty(0, 9, device="cuda"), none, torch.empty(0, 3, device="cuda"))
    assert loss.shape == (0,) and stats.shape == (0, 2)
    assert dec.distill_backward(loss, torch.empty(0, 9, device="cuda"), none, torch.empty(0, 3, device="cuda"), stats).shape == (0, 9)
    s, empty = randn((4, 9), torch.float32, 0), torch.empty(4, 0, device="cuda")
    loss, stats = dec.distill_forward(s, empty.long(), empty)   # lists of no length
    assert not loss.any() and not dec.distill_backward(loss, s, empty.long(), empty, stats).any()
    loss, _ = dec.distill_forward(torch.empty(2, 0, device="cuda"), torch.full((2, 1), -1, device="cuda"), torch.zeros(2, 1, device="cuda"))
    assert not loss.any()


def test_distill_gradient_writes_its_rows_only(ampq, dec):
    s, index, teacher = randn((5, 77), torch.bfloat16, 1), lists(5, 77, 4, 2), randn((5, 4), torch.float32, 3)
    loss, stats = dec.distill_forward(s, index, teacher)
    full = torch.full((6, 101), 5.0, dtype=torch.bfloat16, device="cuda")
    gl, st = torch.ones(5, device="cuda"), torch.cuda.current_stream().cuda_stream
    rc = ampq.lib().ampq_distill_backward(0, st, ampq.BF16, ampq.F32, ampq.I64, gl.data_ptr(), 1, s.data_ptr(), 77, 5, 77, index.data_ptr(), 4, teacher.data_ptr(), 4, 4,
                                          stats.data_ptr(), 1.0, full.data_ptr() + 2 * 11, 101)
    assert rc == 0 and torch.equal(full[:5, 11:88], dec.distill_backward(gl, s, index, teacher, stats))
    full[:5, 11:88] = 5.0
    assert bool((full == 5.0).all())


def test_distill_repeats_itself(dec):
    s, index, teacher = randn((3, 90000), torch.bfloat16, 4, 2.0), lists(3, 90000, 64, 5, ragged=False), randn((3, 64), torch.float32, 6)
    first = dec.distill_forward(s, index, teacher)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, dec.distill_forward(s, index, teacher)))


@pytest.mark.parametrize("n", [129, 144, 300, 8192, 8193, 40000])
def test_embed_grad_of_one_run(dec, n):
    """Runs of 9 pieces and more, which are added up in groups: one token for all but a few, over several blocks of columns."""
    tokens = torch.full((n,), 5)
    tokens[::97] = 2
    check_embed_grad(dec, tokens.cuda(), randn((n, 24), torch.float32, n), 7, 1.0)
    if n < 10000:
        check_embed_grad(dec, tokens.cuda(), randn((n, 1100), torch.bfloat16, n), 7, 1.0)
        check_embed_grad(dec, tokens.cuda(), randn((n, 523), torch.float32, n), 7, 1.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_distill_of_repeated_columns(dec, dtype):
    """Long lists with columns listed many times over, the row's first and last columns among them, in rows of one part and
    of several."""
    for rows, cols, top, seed in [(6, 45, 900, 1), (5, 50021, 1024, 2), (4, 70007, 129, 3), (3, 40, 128, 4)]:
        s = randn((rows, cols), dtype, seed, 2.0)
        index = lists(rows, cols, top, seed)
        index[:, ::7] = 0
        index[:, 3::7] = cols - 1
        index[0, 1::7] = cols // 2
        check_distill(dec, s, index, randn((rows, top), torch.float32, seed + 10), 1.0)
