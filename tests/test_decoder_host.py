"""Refusals of the embedding, head norm and distillation calls, and the gradients of their definitions against
differences: nothing here needs a GPU (arguments are looked at before a device is)."""
import ctypes as C

import numpy as np
import pytest
import torch

import decoder_reference as ref

A = 1 << 20  # an aligned address that nothing reads: every call here is refused before it launches
BIG = 1 << 31


def embed(L, dtype=0, index=0, tokens=A, n=4, w=A, ldw=40, vocab=9, cols=40, scale=1.0, y=A, ldy=40):
    return L.ampq_embed_forward(0, None, dtype, index, tokens, n, w, ldw, vocab, cols, scale, y, ldy)


def embed_back(L, dtype=0, index=0, tokens=A, n=4, gy=A, ldg=40, vocab=9, cols=40, scale=1.0, padding=-1, gw=A, ws=A, size=1 << 30):
    return L.ampq_embed_backward(0, None, dtype, index, tokens, n, gy, ldg, vocab, cols, scale, padding, gw, ws, size)


def side(L, heads=2, x=A, xs=(320, 80, 40), gy=A, gs=(320, 80, 40), out=A, os=(320, 80, 40), w=A, gw=A, rstd=A, codes=A, ldc=64, scales=A, lds=2):
    from paper_2505_13060_b200 import binding

    return C.byref(binding.Heads(heads, x, *xs, gy, *gs, out, *os, w, gw, rstd, codes, ldc, scales, lds))


def heads(L, dtype=0, pdtype=0, index=0, fmt=1, batch=3, tokens=4, cols=40, rot=20, cos=A, sin=A, angles=64, pos=A, ps=0, eps=1e-5, q={}, k={}, no_q=False):
    return L.ampq_head_norm_forward(0, None, dtype, pdtype, index, fmt, 0, batch, tokens, cols, rot, cos, sin, angles, pos, ps, eps,
                                    None if no_q else side(L, **q), side(L, **k))


def heads_back(L, dtype=0, pdtype=0, index=0, fmt=1, batch=3, tokens=4, cols=40, rot=20, cos=A, sin=A, angles=64, pos=A, ps=0, q={}, k={}, ws=A, size=1 << 30):
    return L.ampq_head_norm_backward(0, None, dtype, pdtype, index, fmt, 0, batch, tokens, cols, rot, cos, sin, angles, pos, ps, side(L, **q), side(L, **k), ws,
                                     size)


def distill(L, dtype=0, tdtype=0, index=0, s=A, ld=40, rows=4, cols=40, idx=A, ldi=5, t=A, ldt=5, top=5, T=1.0, loss=A, stats=A):
    return L.ampq_distill_forward(0, None, dtype, tdtype, index, s, ld, rows, cols, idx, ldi, t, ldt, top, T, loss, stats)


def distill_back(L, dtype=0, tdtype=0, index=0, gl=A, gls=1, s=A, ld=40, rows=4, cols=40, idx=A, ldi=5, t=A, ldt=5, top=5, stats=A, T=1.0, gs=A, ldg=40):
    return L.ampq_distill_backward(0, None, dtype, tdtype, index, gl, gls, s, ld, rows, cols, idx, ldi, t, ldt, top, stats, T, gs, ldg)


LISTS = [dict(dtype=2), dict(tdtype=2), dict(index=2), dict(index=-1), dict(s=0), dict(rows=-1), dict(cols=-1), dict(ld=39), dict(idx=0), dict(t=0),
         dict(top=-1), dict(ldi=4), dict(ldt=4), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-7), dict(T=2e6)]
HEADS = [dict(dtype=2), dict(pdtype=-1), dict(index=2), dict(fmt=3), dict(batch=-1), dict(tokens=-1), dict(cols=-2), dict(cols=39), dict(rot=-2), dict(rot=19),
         dict(rot=42), dict(cos=0), dict(sin=0), dict(angles=-1), dict(ps=-1), dict(q=dict(heads=-1)), dict(k=dict(heads=-1)), dict(q=dict(out=0)),
         dict(k=dict(rstd=0)), dict(q=dict(xs=(-1, 80, 40))), dict(q=dict(os=(320, 80, -40))), dict(k=dict(gs=(1 << 41, 0, 0))),
         dict(q=dict(codes=0)), dict(q=dict(ldc=32)), dict(k=dict(lds=1))]
HEADS_ALIGN = [dict(cos=A + 4), dict(sin=A + 8), dict(pos=A + 2), dict(index=1, pos=A + 4), dict(q=dict(x=A + 2)), dict(k=dict(out=A + 2)), dict(q=dict(w=A + 2)),
               dict(q=dict(rstd=A + 2)), dict(q=dict(codes=A + 8)), dict(k=dict(ldc=72))]
HEADS_LARGE = [dict(cols=258, rot=0, q=dict(ldc=288, lds=9), k=dict(ldc=288, lds=9)), dict(batch=BIG), dict(batch=1 << 16, tokens=1 << 16), dict(q=dict(heads=1 << 21)),
               dict(batch=1 << 12, tokens=1 << 12, k=dict(heads=1 << 10)), dict(angles=BIG)]
REFUSED = [
    (embed, "INVALID", [dict(dtype=2), dict(index=2), dict(tokens=0), dict(n=-1), dict(vocab=-1), dict(cols=-1), dict(w=0), dict(y=0), dict(ldw=39), dict(ldy=39)]),
    (embed, "ALIGN", [dict(tokens=A + 2), dict(index=1, tokens=A + 4), dict(w=A + 2), dict(y=A + 1)]),
    (embed, "TOO_LARGE", [dict(n=BIG), dict(vocab=BIG), dict(cols=1 << 30, ldw=1 << 30, ldy=1 << 30), dict(ldw=1 << 41)]),
    (embed_back, "INVALID", [dict(dtype=-1), dict(index=3), dict(tokens=0), dict(n=-1), dict(vocab=-1), dict(cols=-1), dict(gy=0), dict(gw=0), dict(ldg=39)]),
    (embed_back, "ALIGN", [dict(tokens=A + 1), dict(gy=A + 2), dict(gw=A + 2), dict(ws=A + 16)]),
    (embed_back, "TOO_LARGE", [dict(n=BIG), dict(vocab=BIG), dict(vocab=BIG - 1, cols=1 << 29, ldg=1 << 29)]),
    (heads, "INVALID", HEADS + [dict(q=dict(x=0)), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(no_q=True)]),
    (heads, "ALIGN", HEADS_ALIGN),
    (heads, "TOO_LARGE", HEADS_LARGE),
    (heads_back, "INVALID", HEADS + [dict(q=dict(gy=0)), dict(fmt=0, k=dict(x=0))]),
    (heads_back, "ALIGN", HEADS_ALIGN + [dict(k=dict(gy=A + 2)), dict(q=dict(gw=A + 2)), dict(ws=A + 128)]),
    (heads_back, "TOO_LARGE", HEADS_LARGE),
    (distill, "INVALID", LISTS + [dict(loss=0), dict(stats=0)]),
    (distill, "ALIGN", [dict(s=A + 2), dict(dtype=1, s=A + 1), dict(idx=A + 2), dict(index=1, idx=A + 4), dict(t=A + 2), dict(loss=A + 2), dict(stats=A + 1)]),
    (distill, "TOO_LARGE", [dict(top=1025, ldi=1025, ldt=1025), dict(rows=BIG), dict(cols=1 << 30, ld=1 << 30), dict(ldi=1 << 41), dict(ldt=1 << 41)]),
    (distill_back, "INVALID", LISTS + [dict(gl=0), dict(gls=-1), dict(stats=0), dict(gs=0), dict(ldg=39)]),
    (distill_back, "ALIGN", [dict(s=A + 2), dict(gs=A + 2), dict(gl=A + 2), dict(stats=A + 2), dict(idx=A + 1), dict(t=A + 1)]),
    (distill_back, "TOO_LARGE", [dict(top=1025, ldi=1025, ldt=1025), dict(gls=1 << 41), dict(ldg=1 << 41)]),
]


@pytest.mark.parametrize("call,status,changes", REFUSED, ids=["%s-%s" % (c.__name__, s) for c, s, _ in REFUSED])
def test_refusals(ampq, call, status, changes):
    for change in changes:
        assert call(ampq.lib(), **change) == getattr(ampq, "ERR_" + status), change


def test_workspace_queries_refuse(ampq):
    L, n = ampq.lib(), C.c_longlong()
    assert L.ampq_embed_backward_workspace(0, 0, 4, 9, 40, None) == ampq.ERR_INVALID
    assert L.ampq_embed_backward_workspace(0, 2, 4, 9, 40, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_embed_backward_workspace(0, 0, -1, 9, 40, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_embed_backward_workspace(0, 0, BIG, 9, 40, C.byref(n)) == ampq.ERR_TOO_LARGE
    assert L.ampq_embed_backward_workspace(0, 0, 4, BIG, 40, C.byref(n)) == ampq.ERR_TOO_LARGE
    assert L.ampq_head_norm_backward_workspace(0, 1, 4, 40, None) == ampq.ERR_INVALID
    assert L.ampq_head_norm_backward_workspace(0, -1, 4, 40, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_head_norm_backward_workspace(0, 1, 4, 41, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_head_norm_backward_workspace(0, 1, 4, 258, C.byref(n)) == ampq.ERR_TOO_LARGE
    assert L.ampq_head_norm_backward_workspace(0, 1 << 16, 1 << 16, 40, C.byref(n)) == ampq.ERR_TOO_LARGE


def test_no_device_is_an_error(ampq):
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    L, n = ampq.lib(), C.c_longlong()
    assert {c(L) for c in (embed, embed_back, heads, heads_back, distill, distill_back)} == {ampq.ERR_CUDA}
    assert L.ampq_embed_backward_workspace(0, 0, 4, 9, 40, C.byref(n)) == ampq.ERR_CUDA
    assert L.ampq_head_norm_backward_workspace(0, 1, 4, 40, C.byref(n)) == ampq.ERR_CUDA


def test_tensors_are_checked(ampq):
    from paper_2505_13060_b200 import decoder as dec

    w, x, i = torch.zeros(9, 40), torch.zeros(3, 2, 40), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: dec.embed(i, w), lambda: dec.embed_backward(i, w[:3], 9), lambda: dec.head_norm_forward(x, None),
                 lambda: dec.distill_forward(w, torch.zeros(9, 2, dtype=torch.int64), torch.zeros(9, 2))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="rows and columns"):
        dec.embed(i, w[0])
    with pytest.raises(ValueError, match="each token"):
        dec.embed_backward(i, w, 9)
    with pytest.raises(ValueError, match="padding_idx"):
        dec.embed_backward(i, w[:3], 9, padding_idx=9)
    with pytest.raises(ValueError, match="heads, columns"):
        dec.head_norm_forward(w, None)
    with pytest.raises(ValueError, match="each row"):
        dec.distill_forward(w, torch.zeros(8, 2, dtype=torch.int64), torch.zeros(8, 2))
    with pytest.raises(ValueError, match="each row"):
        dec.distill_forward(w, torch.zeros(9, 2, dtype=torch.int64), torch.zeros(9, 3))
    with pytest.raises(ValueError, match="constant"):
        dec.distill_loss(w, torch.zeros(9, 2, dtype=torch.int64), torch.zeros(9, 2, requires_grad=True))
    with pytest.raises(ValueError, match="pairs"):
        dec.rotary_table(4, 3, device="cpu")


def test_rotary_table():
    """Angles of far positions, whose products an fp32 angle would lose."""
    from paper_2505_13060_b200 import decoder as dec

    cos, sin = dec.rotary_table(100000, 16, 500000.0, device="cpu")
    angle = np.arange(100000)[:, None] * 500000.0 ** (-np.arange(8) / 8.0)
    # half a step of fp32, and what 64 bits lose of an angle below 2^17 in its power and product
    assert np.abs(cos.double().numpy() - np.cos(angle)).max() <= 2.0 ** -24 * (1 + 1e-3)
    assert np.abs(sin.double().numpy() - np.sin(angle)).max() <= 2.0 ** -24 * (1 + 1e-3)
    assert dec.rotary_table(5, 0, device="cpu")[0].shape == (5, 0)


# -- the definitions' gradients against differences ------------------------------------------------------------------


def differences(f, x, step=1e-6):
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        g[i] = (f(up) - f(down)) / (2 * step)
    return g


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 4, 10])
def test_head_norm_differences(rot, interleaved):
    rng = np.random.default_rng(rot)
    x, w, gy = rng.standard_normal((2, 3, 2, 10)), rng.standard_normal(10), rng.standard_normal((2, 3, 2, 10))
    angle = rng.uniform(0, 6, (2, 3, rot // 2))
    cos, sin = np.cos(angle), np.sin(angle)
    rstd = ref.head_norm(x, w, cos, sin, rot, 1e-5, interleaved)[2]
    gx, gw = ref.head_norm_grad(gy, x, rstd, w, cos, sin, rot, interleaved)[:2]
    # eps is part of rstd: the formula for gx has rstd, not the mean of squares, so it is exact with it too
    f = lambda x, w: (ref.head_norm(x, w, cos, sin, rot, 1e-5, interleaved)[0] * gy).sum()
    assert np.allclose(gx, differences(lambda v: f(v, w), x), rtol=1e-6, atol=1e-7)
    assert np.allclose(gw, differences(lambda v: f(x, v), w), rtol=1e-6, atol=1e-7)


def test_embed_differences():
    rng = np.random.default_rng(0)
    tokens, w, gy = np.array([3, 0, 3, 1, 3]), rng.standard_normal((5, 4)), rng.standard_normal((5, 4))
    f = lambda w: (0.7 * w[tokens] * gy).sum()
    assert np.allclose(ref.embed_grad(tokens, gy, 5, 0.7)[0], differences(f, w), rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distill_differences(T):
    rng = np.random.default_rng(1)
    s, t = rng.standard_normal((4, 11)), rng.standard_normal((4, 5))
    idx = np.array([[1, 5, 9, 0, 2], [3, -1, 7, 3, 3], [-1, -1, -1, -1, -1], [10, 4, -1, -1, -1]])   # twice the same, none, few
    gl = rng.standard_normal(4)
    g = ref.distill_grad(gl, s, idx, t, T)[0]
    assert np.allclose(g, differences(lambda v: (ref.distill(v, idx, t, T) * gl).sum(), s), rtol=1e-5, atol=1e-7)
    assert ref.distill(s, idx, t, T)[2] == 0 and not g[2].any()
    # a list of all columns with the row's own logits has no divergence
    every = np.tile(np.arange(11), (4, 1))
    assert np.abs(ref.distill(s, every, s, T)).max() < 1e-12
