"""8-bit checkpoints, the weight gradient from them and the norms on the GPU,
against plain 64-bit implementations on the host.

Codes and scale bytes have to be equal.  Sums: an fp32 sum of n products is off
by at most about n * 2^-24 times the sum of the absolute products (each addition
rounds once; a tensor core's additions may cut instead of round: twice that),
plus half a step of the output's type, eps/2 relative.
"""
import numpy as np
import pytest
import torch

import ckpt_reference as ref

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


def laid(t, layout):
    """The same values: as they are, in wider rows that start 16-byte aligned, or in rows that start anywhere."""
    if layout == "plain":
        return t
    extra, at = (64, 0) if layout == "wide" else (3, 1)
    full = torch.full((t.shape[0], t.shape[1] + extra), 7.0, dtype=t.dtype, device=t.device)
    out = full[:, at:at + t.shape[1]]
    out.copy_(t)
    return out


def values(rows, cols, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed * 1000 + rows * 7 + cols)
    x = torch.randn(rows, cols, generator=g) * scale
    x[:, torch.randperm(cols, generator=g)[:max(1, cols // 50)]] *= 50.0
    return x.to(dtype).cuda()


SIZES = [(1, 1), (1, 31), (3, 32), (5, 33), (2, 40), (7, 257), (64, 256), (33, 1001), (3, 4104), (300, 72)]


@pytest.mark.parametrize("layout", ["plain", "wide", "odd"])
@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_pack_and_unpack(ckpt, dtype, fmt, layout):
    for rows, cols in SIZES:
        x = values(rows, cols, dtype, 1)
        p = ckpt.pack(laid(x, layout), fmt)
        codes, scales = ref.pack(f64(x), fmt)
        assert np.array_equal(p.scales.cpu().numpy(), scales), (rows, cols)
        assert np.array_equal(p.codes.cpu().numpy(), codes), (rows, cols)
        for out in DTYPES:
            assert np.array_equal(f64(ckpt.unpack(p, out)), ref.unpack(codes, scales, cols, fmt)), (rows, cols, out)


@pytest.mark.parametrize("fmt", [1, 2])
def test_pack_borders(ckpt, fmt):
    """Every group its own magnitude, from the smallest fp32 to the largest; exact ties; zeros of both signs;
    groups with Inf or NaN."""
    g = ref.grid(fmt)
    rows = []
    for e in list(range(-149, 128, 3)) + [126, 127]:
        rows.append([1.75 * 2.0 ** e * f for f in ((-1.0) ** i * (1 - i / 40) for i in range(32))])
        rows.append([1.7500001 * 2.0 ** e] + [2.0 ** (e - i) for i in range(31)])
    mids = list((g[1:] + g[:-1]) / 2)
    for i in range(0, len(mids), 31):
        rows.append(([g[-1]] + mids[i:i + 31] + [-0.0] * 32)[:32])
    rows += [[0.0] * 32, [-0.0] * 32, [float(np.finfo(np.float32).max)] * 32]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 7, 31):
            r = list(np.linspace(-3, 3, 32))
            r[at] = bad
            rows.append(r)
    x32 = torch.tensor(np.array(rows), dtype=torch.float64).float()
    x32 = torch.cat([x32, x32.roll(1, 0), x32[:, :19]], 1)  # three groups a row, the last one short
    for x in (x32.cuda(), x32.bfloat16().cuda()):
        p = ckpt.pack(x, fmt)
        codes, scales = ref.pack(f64(x), fmt)
        assert np.array_equal(p.scales.cpu().numpy(), scales)
        assert np.array_equal(p.codes.cpu().numpy(), codes)
        for out in DTYPES:
            got = f64(ckpt.unpack(p, out))
            assert np.array_equal(got, ref.unpack(codes, scales, x.shape[1], fmt), equal_nan=True)


def test_pitches_and_what_lies_behind(ampq, ckpt):
    """Wider pitches than needed: bytes behind a row's last group, and outputs behind a row, stay as they were."""
    rows, cols = 9, 75
    x = values(rows, cols, torch.float32, 2)
    st = torch.cuda.current_stream().cuda_stream
    codes = torch.full((rows, 144), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, 7), 0xCD, dtype=torch.uint8, device="cuda")
    L = ampq.lib()
    assert L.ampq_ckpt_pack(0, st, ampq.F32, 1, x.data_ptr(), rows, cols, cols, codes.data_ptr(), 144, scales.data_ptr(), 7) == 0
    want, wscale = ref.pack(f64(x), 1)
    assert np.array_equal(codes[:, :96].cpu().numpy(), want) and bool((codes[:, 96:] == 0xAB).all())
    assert np.array_equal(scales[:, :3].cpu().numpy(), wscale) and bool((scales[:, 3:] == 0xCD).all())
    out = torch.full((rows + 1, cols + 5), 3.0, device="cuda")
    assert L.ampq_ckpt_unpack(0, st, ampq.F32, 1, codes.data_ptr(), 144, scales.data_ptr(), 7, rows, cols, out.data_ptr(), cols + 5) == 0
    assert np.array_equal(f64(out[:rows, :cols]), ref.unpack(want, wscale, cols, 1))
    assert bool((out[:, cols:] == 3.0).all()) and bool((out[rows] == 3.0).all())


# -- weight gradient ------------------------------------------------------------------------------------------------


def wgrad_case(ckpt, dtype, fmt, samples, rows, cols, outs, layout="plain", seed=0):
    x = values(samples * rows, cols, dtype, seed)
    gy = laid((torch.randn(samples * rows, outs, generator=torch.Generator().manual_seed(seed + 5)) * 1e-2).to(dtype).cuda(), layout)
    return ckpt.pack(x, fmt), gy


def check_wgrad(p, gy, samples, gw, gb):
    rows, outs = p.rows // samples, gy.shape[1]
    x = ref.unpack(p.codes.cpu().numpy(), p.scales.cpu().numpy(), p.cols, p.fmt).reshape(samples, rows, p.cols)
    g = f64(gy).reshape(samples, rows, outs)
    want = np.einsum("rnk,rnc->rkc", g, x, optimize=True)
    size = np.einsum("rnk,rnc->rkc", np.abs(g), np.abs(x), optimize=True)
    h = HALF_STEP[gy.dtype]
    off = np.abs(f64(gw) - want)
    assert gw.shape == want.shape and gw.dtype == gy.dtype
    tol = (2 * rows + 8) * U * size * (1 + h) + h * np.abs(want)
    assert (off <= tol).all(), (off / np.maximum(tol, 1e-300)).max()
    if gb is not None:
        off, tol = np.abs(f64(gb) - g.sum(1)), (rows + 8) * U * np.abs(g).sum(1) * (1 + h) + h * np.abs(g.sum(1))
        assert (off <= tol).all()


WGRAD = [  # samples, rows, cols, outs
    (1, 1, 1, 1), (1, 1, 32, 8), (2, 3, 33, 5), (8, 128, 256, 256), (1, 64, 64, 64), (3, 97, 131, 70), (1, 17, 257, 264),
    (2, 200, 520, 129), (1, 1000, 40, 24), (5, 31, 16, 513), (1, 2049, 300, 136), (4, 1, 100, 100),
]


@pytest.mark.parametrize("layout", ["plain", "wide", "odd"])
@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_weight_grad(ckpt, dtype, fmt, layout):
    for samples, rows, cols, outs in WGRAD:
        p, gy = wgrad_case(ckpt, dtype, fmt, samples, rows, cols, outs, layout, 3)
        gw, gb = ckpt.weight_grad(p, gy, samples=samples, bias=True)
        check_wgrad(p, gy, samples, gw, gb)
        again, none = ckpt.weight_grad(p, gy, samples=samples)
        assert none is None and torch.equal(gw, again), (samples, rows, cols, outs)


def test_weight_grad_without_rows_or_columns(ckpt):
    p = ckpt.pack(torch.empty(0, 40, device="cuda"))
    gw, gb = ckpt.weight_grad(p, torch.empty(0, 24, device="cuda"), bias=True)
    assert gw.shape == (1, 24, 40) and not gw.any() and not gb.any()
    p = ckpt.pack(torch.empty(6, 0, device="cuda"))
    gw, gb = ckpt.weight_grad(p, torch.ones(6, 24, device="cuda"), samples=2, bias=True)
    assert gw.shape == (2, 24, 0) and bool((gb == 3).all())
    p = ckpt.pack(torch.ones(6, 24, device="cuda"))
    gw, gb = ckpt.weight_grad(p, torch.empty(6, 0, device="cuda"), samples=2, bias=True)
    assert gw.shape == (2, 0, 24) and gb.shape == (2, 0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_weight_grad_non_finite(ckpt, dtype):
    """An Inf or a NaN reaches exactly the entries it reaches in the formula."""
    samples, rows, cols, outs = 2, 70, 96, 48
    x = values(samples * rows, cols, dtype, 4)
    x[75, 40] = float("nan")   # sample 1, group 1
    x[80, 70] = float("inf")   # sample 1, group 2
    gy = (torch.randn(samples * rows, outs, generator=torch.Generator().manual_seed(6)) + 3).to(dtype).cuda()
    gy[10, 5] = float("inf")   # sample 0
    gy[139, 7] = float("nan")  # sample 1, last row
    p = ckpt.pack(x)
    gw, gb = ckpt.weight_grad(p, gy, samples=samples, bias=True)
    xs = ckpt.unpack(p, torch.float32).double().reshape(samples, rows, cols)
    want = torch.matmul(gy.double().reshape(samples, rows, outs).transpose(1, 2), xs)
    assert torch.equal(torch.isnan(gw), torch.isnan(want))
    assert torch.equal(torch.isinf(gw), torch.isinf(want))
    fine = torch.isfinite(want)
    size = torch.matmul(gy.double().abs().nan_to_num(0, 0).reshape(samples, rows, outs).transpose(1, 2), xs.abs().nan_to_num(0, 0))
    tol = (2 * rows + 8) * U * size + HALF_STEP[dtype] * 1.01 * want.abs()
    assert bool(((gw.double() - want).abs()[fine] <= tol[fine]).all())
    assert torch.equal(torch.isnan(gb), torch.isnan(gy.double().reshape(samples, rows, outs).sum(1)))


# -- norms --------------------------------------------------------------------------------------------------------------

NORM = [(1, 1), (1, 8), (3, 31), (300, 256), (17, 257), (5, 512), (70, 1000), (9, 1024), (6, 2047), (33, 4099), (600, 72),
        (4, 5120), (3, 8192), (2, 8200), (3, 16384)]
DEPTH = 64  # additions on one value's way into a row's sum: at most 32 in a thread, 5 in a warp, 16 or 32 warps


@pytest.mark.parametrize("layout", ["plain", "wide", "odd"])
@pytest.mark.parametrize("kind", [0, 1], ids=["layer", "rms"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_norm_forward(ckpt, dtype, kind, layout):
    for k, (rows, cols) in enumerate(NORM):
        fmt = k % 3
        x = values(rows, cols, dtype, 7) + (0.5 if kind == 0 else 0.0)
        pdtype = DTYPES[k % 2]
        w = (1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(k))).to(pdtype).cuda() if k % 5 != 4 else None
        b = torch.randn(cols, generator=torch.Generator().manual_seed(k + 50)).to(pdtype).cuda() if kind == 0 and k % 4 != 3 else None
        eps = 1e-5
        y, mean, rstd, p = ckpt.norm_forward(laid(x, layout), w, b, eps, kind, fmt)
        v = f64(x)
        m = v.mean(1) if kind == 0 else np.zeros(rows)
        d = v - m[:, None]
        var = (d * d).mean(1)
        r = 1 / np.sqrt(var + eps)
        off_m = (DEPTH + 2) * U * np.abs(v).mean(1) if kind == 0 else np.zeros(rows)
        if kind == 0:
            assert (np.abs(f64(mean) - m) <= off_m).all()
        else:
            assert mean is None
        # the squared differences: off by the mean's error (its square, since they sum to nothing) and a sum's rounding;
        # half of a relative error of the variance reaches rstd, whose own division and root round three times
        rel_r = 0.5 * ((DEPTH + 6) * U + (off_m ** 2 + 2 * U * off_m * np.abs(d).mean(1)) / (var + eps)) * 1.01 + 3 * U
        assert (np.abs(f64(rstd) - r) <= rel_r * r).all()
        wv = f64(w) if w is not None else np.ones(cols)
        bv = f64(b) if b is not None else np.zeros(cols)
        want = d * r[:, None] * wv + bv
        h = HALF_STEP[dtype]
        tol = (np.abs(d) * (rel_r + 4 * U)[:, None] + off_m[:, None]) * r[:, None] * np.abs(wv) * 1.01 + (h + 2 * U) * np.abs(want) + 1e-45
        assert (np.abs(f64(y) - want) <= tol).all(), (rows, cols)
        if fmt:
            codes, scales = ref.pack(v, fmt)
            assert np.array_equal(p.codes.cpu().numpy(), codes) and np.array_equal(p.scales.cpu().numpy(), scales), (rows, cols)
        else:
            assert p is None


@pytest.mark.parametrize("layout", ["plain", "wide", "odd"])
@pytest.mark.parametrize("kind", [0, 1], ids=["layer", "rms"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_norm_backward(ckpt, dtype, kind, layout):
    for k, (rows, cols) in enumerate(NORM):
        fmt = k % 3
        x = values(rows, cols, dtype, 8) + (0.5 if kind == 0 else 0.0)
        pdtype = DTYPES[(k // 2) % 2]
        w = (1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(k))).to(pdtype).cuda() if k % 5 != 4 else None
        gy = (torch.randn(rows, cols, generator=torch.Generator().manual_seed(k + 9)) * 1e-2).to(dtype).cuda()
        _, mean, rstd, p = ckpt.norm_forward(x, w, None, 1e-5, kind, fmt)
        kept = p if fmt else laid(x, layout)
        gx, gw, gb = ckpt.norm_backward(laid(gy, layout), kept, mean, rstd, w, kind)
        v = ref.unpack(p.codes.cpu().numpy(), p.scales.cpu().numpy(), cols, fmt) if fmt else f64(x)
        g, r = f64(gy), f64(rstd)[:, None]
        h = (v - (f64(mean)[:, None] if kind == 0 else 0.0)) * r
        wv = f64(w) if w is not None else np.ones(cols)
        t = g * wv
        c2 = (t * h).mean(1, keepdims=True)
        c1 = t.mean(1, keepdims=True) if kind == 0 else np.zeros((rows, 1))
        want = r * (t - c1 - h * c2)
        e1 = (DEPTH + 6) * U * np.abs(t).mean(1, keepdims=True) if kind == 0 else 0.0
        e2 = (DEPTH + 10) * U * np.abs(t * h).mean(1, keepdims=True)
        half = HALF_STEP[dtype]
        tol = r * (8 * U * (np.abs(t) + np.abs(c1) + np.abs(h * c2)) + e1 + np.abs(h) * e2) * 1.01 + half * np.abs(want) + 1e-45
        off = np.abs(f64(gx) - want)
        assert gx.dtype == dtype and (off <= tol).all(), (rows, cols, (off / tol).max())
        half = HALF_STEP[pdtype if w is not None else dtype]
        if w is None:
            assert gw is None
        else:
            want = (g * h).sum(0)
            tol = (rows + 8) * U * np.abs(g * h).sum(0) * 1.01 + half * np.abs(want) + 1e-45
            assert gw.dtype == pdtype and (np.abs(f64(gw) - want) <= tol).all(), (rows, cols)
        if kind == 0:
            want = g.sum(0)
            tol = (rows + 8) * U * np.abs(g).sum(0) * 1.01 + half * np.abs(want) + 1e-45
            assert (np.abs(f64(gb) - want) <= tol).all(), (rows, cols)
        else:
            assert gb is None
        again = ckpt.norm_backward(laid(gy, layout), kept, mean, rstd, w, kind)
        assert torch.equal(gx, again[0]) and (gw is None or torch.equal(gw, again[1]))


def test_norm_backward_against_differences(ckpt):
    """The gradient agrees with differences of the forward pass in 64 bits."""
    rows, cols = 3, 70
    for kind in (0, 1):
        x, gy = values(rows, cols, torch.float32, 11), values(rows, cols, torch.float32, 12)
        w = 1 + 0.1 * torch.randn(cols, device="cuda")
        _, mean, rstd, _ = ckpt.norm_forward(x, w, None, 1e-5, kind)
        gx, gw, _ = ckpt.norm_backward(gy, x, mean, rstd, w, kind)

        def loss(v, u):
            d = v - v.mean(1, keepdims=True) if kind == 0 else v
            return (f64(gy) * d / np.sqrt((d * d).mean(1, keepdims=True) + 1e-5) * u).sum()

        v, u, step = f64(x), f64(w), 1e-6
        rng = np.random.default_rng(3)
        for _ in range(5):
            dv, du = rng.standard_normal(v.shape), rng.standard_normal(u.shape)
            diff = (loss(v + step * dv, u + step * du) - loss(v - step * dv, u - step * du)) / (2 * step)
            got = (f64(gx) * dv).sum() + (f64(gw) * du).sum()
            size = np.abs(f64(gx) * dv).sum() + np.abs(f64(gw) * du).sum()
            assert abs(got - diff) <= 1e-5 * size


def test_norm_empty_and_zero_rows(ckpt):
    w = torch.ones(48, device="cuda")
    y, mean, rstd, p = ckpt.norm_forward(torch.empty(0, 48, device="cuda"), w, w, 1e-5, 0, 1)
    assert y.shape == (0, 48) and p.rows == 0
    gx, gw, gb = ckpt.norm_backward(torch.empty(0, 48, device="cuda"), p, mean, rstd, w, 0)
    assert gx.shape == (0, 48) and not gw.any() and not gb.any()
    y, mean, rstd, p = ckpt.norm_forward(torch.zeros(4, 48, device="cuda"), w, w, 1e-5, 0, 1)
    assert bool((y == 1).all()) and bool((p.scales == 127).all()) and not p.codes.any()
    bad = torch.zeros(4, 48, device="cuda")
    bad[1, 3] = float("nan")
    y, mean, rstd, p = ckpt.norm_forward(bad, w, w, 1e-5, 0, 1)
    assert bool(torch.isnan(y[1]).all()) and bool((y[[0, 2, 3]] == 1).all()) and int(p.scales[1, 0]) == 255


# -- streams, graphs -----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_captured_and_replayed(ckpt, dtype):
    """The whole set in one graph on another stream, replayed on new inputs: the same bits as called one by one."""
    samples, rows, cols, outs = 2, 150, 264, 136
    n = samples * rows
    x, gy, gz = values(n, cols, dtype, 20), values(n, outs, dtype, 21), values(n, cols, dtype, 22)
    w = torch.rand(cols, device="cuda").to(dtype)
    b = torch.rand(cols, device="cuda").to(dtype)

    def passes():
        y, mean, rstd, px = ckpt.norm_forward(x, w, b, 1e-5, 0, 1)
        py = ckpt.pack(y, 2)
        gw, gb = ckpt.weight_grad(py, gy, samples=samples, bias=True)
        return [y, ckpt.unpack(py, dtype), gw, gb, *ckpt.norm_backward(gz, px, mean, rstd, w, 0)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        passes()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs_ = passes()
    for seed in (30, 31):
        x.copy_(values(n, cols, dtype, seed))
        gy.copy_(values(n, outs, dtype, seed + 5))
        gz.copy_(values(n, cols, dtype, seed + 9))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(outs_, passes()):
            assert torch.equal(a, c)


def test_two_streams_at_once(ckpt):
    """Calls that overlap on two streams do not see each other."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    cases = [wgrad_case(ckpt, torch.bfloat16, 1, 2, 700, 320, 520, seed=s) for s in (40, 41)]
    alone = [ckpt.weight_grad(p, gy, samples=2, bias=True) for p, gy in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate((a, b)):
            with torch.cuda.stream(s):
                got[k].append(ckpt.weight_grad(*cases[k], samples=2, bias=True))
    torch.cuda.synchronize()
    for k in range(2):
        for gw, gb in got[k]:
            assert torch.equal(gw, alone[k][0]) and torch.equal(gb, alone[k][1])


# More rows than the row groups of a grid: every group works through several, with copies of the next ones on their way.
MANY = [(9700, 40), (9600, 256), (5200, 1000), (3000, 2048), (1900, 3000), (1400, 4096), (1300, 5120), (900, 4099), (1400, 8192), (650, 9000), (640, 16384)]


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("kind", [0, 1], ids=["layer", "rms"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_norms_of_many_rows(ckpt, dtype, kind, layout):
    """The same bounds as for few rows, against 64 bits on the device; every row and column is compared."""
    for k, (rows, cols) in enumerate(MANY):
        fmt = (0, 1, 2, 1)[(k + kind) % 4]
        g = torch.Generator(device="cuda").manual_seed(rows + cols)
        x = laid((torch.randn(rows, cols, device="cuda", generator=g) + 0.25 * (1 - kind)).to(dtype), layout)
        gy = laid((torch.randn(rows, cols, device="cuda", generator=g) * 1e-2).to(dtype), layout)
        w = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(dtype)
        b = torch.randn(cols, device="cuda", generator=g).to(dtype) if kind == 0 else None
        y, mean, rstd, p = ckpt.norm_forward(x, w, b, 1e-5, kind, fmt)
        v = x.double()
        m = v.mean(1, keepdim=True) if kind == 0 else torch.zeros(rows, 1, device="cuda", dtype=torch.float64)
        d = v - m
        var = (d * d).mean(1, keepdim=True)
        r = (var + 1e-5).rsqrt()
        off_m = (DEPTH + 2) * U * v.abs().mean(1, keepdim=True) if kind == 0 else torch.zeros_like(m)
        if kind == 0:
            assert bool(((mean[:, None] - m).abs() <= off_m).all()), (rows, cols)
        rel_r = 0.5 * ((DEPTH + 6) * U + (off_m ** 2 + 2 * U * off_m * d.abs().mean(1, keepdim=True)) / (var + 1e-5)) * 1.01 + 3 * U
        assert bool(((rstd[:, None] - r).abs() <= rel_r * r).all()), (rows, cols)
        wd, h = w.double(), HALF_STEP[dtype]
        want = d * r * wd + (b.double() if b is not None else 0.0)
        tol = (d.abs() * (rel_r + 4 * U) + off_m) * r * wd.abs() * 1.01 + (h + 2 * U) * want.abs() + 1e-45
        assert bool(((y.double() - want).abs() <= tol).all()), (rows, cols)
        if fmt:
            q = ckpt.pack(x, fmt)
            assert torch.equal(p.codes, q.codes) and torch.equal(p.scales, q.scales), (rows, cols)
        # the backward pass from what the forward pass left
        gx, gw, gb = ckpt.norm_backward(gy, p if fmt else x, mean, rstd, w, kind)
        v = ckpt.unpack(p, torch.float32).double() if fmt else v
        gd, r = gy.double(), rstd.double()[:, None]
        hn = (v - (mean.double()[:, None] if kind == 0 else 0.0)) * r
        t = gd * wd
        c2 = (t * hn).mean(1, keepdim=True)
        c1 = t.mean(1, keepdim=True) if kind == 0 else torch.zeros_like(c2)
        want = r * (t - c1 - hn * c2)
        e1 = (DEPTH + 6) * U * t.abs().mean(1, keepdim=True) if kind == 0 else 0.0
        e2 = (DEPTH + 10) * U * (t * hn).abs().mean(1, keepdim=True)
        tol = r * (8 * U * (t.abs() + c1.abs() + (hn * c2).abs()) + e1 + hn.abs() * e2) * 1.01 + h * want.abs() + 1e-45
        assert bool(((gx.double() - want).abs() <= tol).all()), (rows, cols)
        # the sums: at most all rows one after the other
        want = (gd * hn).sum(0)
        assert bool(((gw.double() - want).abs() <= (rows + 8) * U * (gd * hn).abs().sum(0) * 1.01 + h * want.abs() + 1e-45).all()), (rows, cols)
        if kind == 0:
            want = gd.sum(0)
            assert bool(((gb.double() - want).abs() <= (rows + 8) * U * gd.abs().sum(0) * 1.01 + h * want.abs() + 1e-45).all()), (rows, cols)


LARGE = [(1, 700, 2600, 2500), (3, 600, 1700, 2300), (2, 4096, 520, 264), (1, 130, 4100, 2100), (5, 300, 1024, 1024)]


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_weight_grad_of_many_tiles(ckpt, dtype, layout):
    """More tiles than the grid, pairs of CTAs, parts of the token axis: against 64 bits on the device."""
    for k, (samples, rows, cols, outs) in enumerate(LARGE):
        p, gy = wgrad_case(ckpt, dtype, 1 + k % 2, samples, rows, cols, outs, layout, 9)
        gw, gb = ckpt.weight_grad(p, gy, samples=samples, bias=True)
        x = ckpt.unpack(p, torch.float32).double().reshape(samples, rows, cols)
        g = gy.double().reshape(samples, rows, outs)
        want, size = torch.matmul(g.transpose(1, 2), x), torch.matmul(g.abs().transpose(1, 2), x.abs())
        h = HALF_STEP[dtype]
        assert bool(((gw.double() - want).abs() <= (2 * rows + 8) * U * size * (1 + h) + h * want.abs()).all()), (samples, rows, cols, outs)
        want = g.sum(1)
        assert bool(((gb.double() - want).abs() <= (rows + 8) * U * g.abs().sum(1) * (1 + h) + h * want.abs()).all())
        again, _ = ckpt.weight_grad(p, gy, samples=samples)
        assert torch.equal(gw, again)


def test_weight_grad_fp32_does_not_drift(ckpt):
    """Sums of one sign over 8192 tokens in fp32: a sum that is cut at every addition would be off by 4e-5 of itself; rounded
    to nearest after each 64 tokens it stays within the sixteen additions of a run (cut: 2^-23 each) and 128 roundings."""
    x = torch.rand(8192, 256, device="cuda") + 0.5
    gy = torch.rand(8192, 512, device="cuda") + 0.5
    p = ckpt.pack(x)
    gw, _ = ckpt.weight_grad(p, gy)
    want = torch.matmul(gy.double().T, ckpt.unpack(p, torch.float32).double())
    assert float(((gw[0].double() - want) / want).abs().max()) <= 16 * 2 * U + 128 * U
    assert float(((gw[0].double() - want) / want).mean().abs()) <= 8 * 2 * U


def test_offsets_past_32_bits(ckpt):
    """Matrices of more than 2^32 elements: the last rows come out as they do alone."""
    rows, cols = 70000, 65536
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = values(5, cols, torch.bfloat16, 50)
    x[:-5].fill_(1.0)
    x[-5:] = tail
    p, q = ckpt.pack(x), ckpt.pack(tail)
    assert torch.equal(p.codes[-5:], q.codes) and torch.equal(p.scales[-5:], q.scales)
    del x
    assert torch.equal(ckpt.unpack(p)[-5:], ckpt.unpack(q))
    del p
    # norms: 2^32 elements in rows of 8192
    n = 2 ** 19 + 3
    x = torch.full((n, 8192), 0.5, dtype=torch.bfloat16, device="cuda")
    x[-3:] = values(3, 8192, torch.bfloat16, 51)
    w = torch.rand(8192, device="cuda").bfloat16()
    y, _, rstd, p = ckpt.norm_forward(x, w, None, 1e-5, 1, 1)
    y3, _, rstd3, p3 = ckpt.norm_forward(x[-3:], w, None, 1e-5, 1, 1)
    assert torch.equal(y[-3:], y3) and torch.equal(rstd[-3:], rstd3) and torch.equal(p.codes[-3:], p3.codes)
    gx, _, _ = ckpt.norm_backward(x, p, None, rstd, w, 1)
    gx3, _, _ = ckpt.norm_backward(x[-3:], p3, None, rstd3, w, 1)
    assert torch.equal(gx[-3:], gx3)
    del x, y, gx, p
    # weight gradient: 2^32 gradient elements, all zero but those of the last sample
    samples, rows, cols, outs = 4, 2 ** 18 + 8, 64, 4200
    gy = torch.zeros(samples * rows, outs, dtype=torch.bfloat16, device="cuda")
    gy[-rows:] = 2.0 ** -8
    p = ckpt.pack(torch.ones(samples * rows, cols, device="cuda"))
    gw, gb = ckpt.weight_grad(p, gy, samples=samples, bias=True)
    assert not gw[:-1].any() and not gb[:-1].any()
    assert bool((gw[-1] == torch.tensor(rows * 2.0 ** -8).bfloat16().cuda()).all()) and bool((gb[-1] == gw[-1, 0, 0]).all())


def test_first_call_inside_a_capture(ampq):
    """Nothing has to be called before a capture: a process whose first calls are captured replays them right."""
    import subprocess
    import sys

    code = """
import sys; sys.path.insert(0, %r)
import torch
from paper_2505_13060_b200 import checkpoint as ckpt
for dtype in (torch.bfloat16, torch.float32):
    x, gy = torch.randn(600, 520, device="cuda").to(dtype), torch.randn(600, 1032, device="cuda").to(dtype)
    w = torch.rand(520, device="cuda").to(dtype)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, mean, rstd, p = ckpt.norm_forward(x, w, w, 1e-5, 0, 1)
        out = [y, *ckpt.weight_grad(p, gy, samples=2, bias=True), *ckpt.norm_backward(y, p, mean, rstd, w, 0), ckpt.unpack(p, dtype)]
    graph.replay()
    torch.cuda.synchronize()
    y, mean, rstd, p = ckpt.norm_forward(x, w, w, 1e-5, 0, 1)
    for a, b in zip(out, [y, *ckpt.weight_grad(p, gy, samples=2, bias=True), *ckpt.norm_backward(y, p, mean, rstd, w, 0), ckpt.unpack(p, dtype)]):
        assert torch.equal(a, b)
print("ok")
""" % __file__.rsplit("/tests/", 1)[0]
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=200)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout + r.stderr


def test_tensor_level_refusals(ampq, ckpt):
    x = torch.ones(6, 64, device="cuda")
    p = ckpt.pack(x)
    w = torch.ones(64, device="cuda")
    _, mean, rstd, _ = ckpt.norm_forward(x, w, None, 1e-5)
    for call in (lambda: ckpt.weight_grad(p, torch.ones(5, 8, device="cuda")), lambda: ckpt.weight_grad(p, torch.ones(6, 8, device="cuda"), samples=4),
                 lambda: ckpt.weight_grad(p, torch.ones(6, 8, device="cuda"), samples=0), lambda: ckpt.weight_grad(p, torch.ones(6, 8)),
                 lambda: ckpt.norm_forward(x, torch.ones(63, device="cuda"), None, 1e-5), lambda: ckpt.norm_forward(x, w.cpu(), None, 1e-5),
                 lambda: ckpt.norm_backward(x[:5], p, mean, rstd, w), lambda: ckpt.norm_backward(x, p, None, rstd, w),
                 lambda: ckpt.norm_backward(x, p, mean, rstd.double(), w), lambda: ckpt.pack(torch.ones((), device="cuda")),
                 lambda: ckpt.Packed(p.codes, p.scales, 65, 1), lambda: ckpt.Packed(p.codes[:3], p.scales, 64, 1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ckpt.pack(x.half()), lambda: ckpt.unpack(p, torch.float16), lambda: ckpt.weight_grad(p, x.double()),
                 lambda: ckpt.norm_forward(x, w.half(), None, 1e-5), lambda: ckpt.norm_forward(x, w, w.bfloat16(), 1e-5),
                 lambda: ckpt.norm_backward(x, x.bfloat16(), mean, rstd, w)):
        with pytest.raises(TypeError):
            call()
    odd = torch.empty(6, 72, dtype=torch.uint8, device="cuda")
    for call, status in ((lambda: ckpt.unpack(ckpt.Packed(odd, p.scales, 64, 1)), ampq.ERR_ALIGN), (lambda: ckpt.pack(x, 0), ampq.ERR_INVALID),
                         (lambda: ckpt.norm_forward(torch.ones(2, 16385, device="cuda"), None, None, 1e-5), ampq.ERR_TOO_LARGE),
                         (lambda: ckpt.norm_forward(x, w, None, -1.0), ampq.ERR_INVALID)):
        with pytest.raises(ampq.AmpqError) as e:
            call()
        assert e.value.status == status


@pytest.mark.parametrize("pitch", [0, 16, 3], ids=["same", "wide", "odd"])
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_norm_outputs_in_wider_rows(ampq, ckpt, dtype, pitch):
    """Outputs of the C calls in rows of their own pitch: the values of contiguous outputs, and nothing behind a row, behind
    the last row or in front of the first is written."""
    L, st, code = ampq.lib(), torch.cuda.current_stream().cuda_stream, 0 if dtype == torch.float32 else 1
    for rows, cols in ((5, 40), (2500, 64), (700, 4096), (40, 4099), (300, 1001), (310, 5121)):
        x, gy = values(rows, cols, dtype, 60), values(rows, cols, dtype, 61, 1e-2)
        w, b = torch.rand(cols, device="cuda").to(dtype), torch.rand(cols, device="cuda").to(dtype)
        y, mean, rstd, _ = ckpt.norm_forward(x, w, b, 1e-5, 0)
        gx, gw, gb = ckpt.norm_backward(gy, x, mean, rstd, w, 0)
        ld = cols + pitch

        def room():
            return torch.full((rows + 2, ld), 9.0, dtype=dtype, device="cuda")

        def inside(t):
            inner = t[1:rows + 1, :cols]
            rest = torch.ones(t.shape, dtype=torch.bool, device="cuda")
            rest[1:rows + 1, :cols] = False
            assert bool((t[rest] == 9.0).all()), (rows, cols)
            return inner

        t = room()
        assert L.ampq_norm_forward(0, st, 0, code, code, 0, x.data_ptr(), cols, rows, cols, w.data_ptr(), b.data_ptr(), 1e-5, t[1].data_ptr(), ld,
                                   mean.data_ptr(), rstd.data_ptr(), 0, 0, 0, 0) == 0
        assert torch.equal(inside(t), y)
        t, ws = room(), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        gw2, gb2 = torch.empty_like(gw), torch.empty_like(gb)
        assert L.ampq_norm_backward(0, st, 0, code, code, 0, gy.data_ptr(), cols, x.data_ptr(), cols, 0, 0, 0, 0, rows, cols, mean.data_ptr(),
                                    rstd.data_ptr(), w.data_ptr(), t[1].data_ptr(), ld, gw2.data_ptr(), gb2.data_ptr(), ws.data_ptr(), ws.numel()) == 0
        assert torch.equal(inside(t), gx) and torch.equal(gw, gw2) and torch.equal(gb, gb2)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_weight_grad_writes_its_outputs_only(ampq, ckpt, dtype):
    """Exactly the outputs are written, and every row of gY counts once, whatever boundary it starts on."""
    L, st, code = ampq.lib(), torch.cuda.current_stream().cuda_stream, 0 if dtype == torch.float32 else 1
    for samples, rows, cols, outs, at in ((2, 300, 40, 1301, 0), (1, 611, 130, 515, 1), (3, 1000, 65, 2050, 1), (2, 33, 33, 5, 1), (1, 2000, 24, 513, 3)):
        p, base = wgrad_case(ckpt, dtype, 1, samples, rows, cols, outs, "plain", 70)
        flat = torch.full((samples * rows * (outs + 1) + 8,), 5.0, dtype=dtype, device="cuda")
        gy = flat[at:at + samples * rows * (outs + 1)].view(samples * rows, outs + 1)[:, :outs]
        gy.copy_(base)
        room = [torch.full((k + 64,), 9.0, dtype=dtype, device="cuda") for k in (samples * outs * cols, samples * outs)]
        ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        assert L.ampq_ckpt_weight_grad(0, st, code, 1, gy.data_ptr(), outs + 1, p.codes.data_ptr(), p.codes.stride(0), p.scales.data_ptr(), p.scales.stride(0),
                                       samples, rows, cols, outs, room[0][32:].data_ptr(), room[1][32:].data_ptr(), ws.data_ptr(), ws.numel()) == 0
        for t in room:
            assert bool((t[:32] == 9.0).all()) and bool((t[-32:] == 9.0).all())
        check_wgrad(p, gy, samples, room[0][32:-32].view(samples, outs, cols), room[1][32:-32].view(samples, outs))
