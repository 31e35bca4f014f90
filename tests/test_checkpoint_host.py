"""Refusals of the 8-bit checkpoint and norm calls, and the definition's own
properties: nothing here needs a GPU (arguments are looked at before a device is)."""
import ctypes as C

import numpy as np
import pytest
import torch

import ckpt_reference as ref

A = 1 << 20  # an aligned address that nothing reads: every call here is refused before it launches


def pack(L, dtype=0, fmt=1, x=A, rows=4, cols=40, ld=40, codes=A, ldc=64, scales=A, lds=2):
    return L.ampq_ckpt_pack(0, None, dtype, fmt, x, rows, cols, ld, codes, ldc, scales, lds)


def unpack(L, dtype=0, fmt=1, codes=A, ldc=64, scales=A, lds=2, rows=4, cols=40, out=A, ld=40):
    return L.ampq_ckpt_unpack(0, None, dtype, fmt, codes, ldc, scales, lds, rows, cols, out, ld)


def wgrad(L, dtype=0, fmt=1, gy=A, ldg=24, codes=A, ldc=64, scales=A, lds=2, samples=2, rows=4, cols=40, outs=24, gw=A, gb=0, ws=A, n=1 << 30):
    return L.ampq_ckpt_weight_grad(0, None, dtype, fmt, gy, ldg, codes, ldc, scales, lds, samples, rows, cols, outs, gw, gb, ws, n)


def forward(L, kind=0, dtype=0, pdtype=0, fmt=1, x=A, ldx=40, rows=4, cols=40, w=A, b=A, eps=1e-5, y=A, ldy=40, mean=A, rstd=A,
            codes=A, ldc=64, scales=A, lds=2):
    return L.ampq_norm_forward(0, None, kind, dtype, pdtype, fmt, x, ldx, rows, cols, w, b, eps, y, ldy, mean, rstd, codes, ldc, scales, lds)


def backward(L, kind=0, dtype=0, pdtype=0, fmt=1, gy=A, ldg=40, x=0, ldx=0, codes=A, ldc=64, scales=A, lds=2, rows=4, cols=40, mean=A,
             rstd=A, w=A, gx=A, ldgx=40, gw=A, gb=A, ws=A, n=1 << 30):
    return L.ampq_norm_backward(0, None, kind, dtype, pdtype, fmt, gy, ldg, x, ldx, codes, ldc, scales, lds, rows, cols, mean, rstd, w, gx,
                                ldgx, gw, gb, ws, n)


BIG = 1 << 31
REFUSED = [
    (pack, "INVALID", [dict(dtype=2), dict(dtype=-1), dict(fmt=0), dict(fmt=3), dict(x=0), dict(rows=-1), dict(cols=-1), dict(ld=39),
                       dict(codes=0), dict(scales=0), dict(ldc=48), dict(lds=1)]),
    (pack, "ALIGN", [dict(x=A + 2), dict(dtype=1, x=A + 1), dict(codes=A + 8), dict(ldc=72)]),
    (pack, "TOO_LARGE", [dict(rows=BIG), dict(cols=1 << 30, ld=1 << 30, ldc=1 << 30, lds=1 << 25), dict(ld=1 << 41), dict(ldc=1 << 41)]),
    (unpack, "INVALID", [dict(dtype=2), dict(fmt=0), dict(out=0), dict(codes=0), dict(scales=0), dict(ld=39), dict(lds=1), dict(ldc=32)]),
    (unpack, "ALIGN", [dict(out=A + 1), dict(codes=A + 4)]),
    (wgrad, "INVALID", [dict(dtype=5), dict(fmt=0), dict(gy=0), dict(ldg=23), dict(samples=-1), dict(rows=-1), dict(outs=-1), dict(cols=-1),
                        dict(gw=0), dict(codes=0), dict(scales=0), dict(ldc=32)]),
    (wgrad, "ALIGN", [dict(gy=A + 2), dict(gw=A + 2), dict(gb=A + 1), dict(ws=A + 16), dict(codes=A + 1)]),
    (wgrad, "TOO_LARGE", [dict(samples=1 << 20, rows=1 << 20), dict(outs=1 << 30, ldg=1 << 30)]),
    (forward, "INVALID", [dict(kind=2), dict(dtype=2), dict(pdtype=2), dict(fmt=3), dict(x=0), dict(y=0), dict(ldx=39), dict(ldy=39),
                          dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(mean=0), dict(rstd=0), dict(kind=1),
                          dict(codes=0), dict(lds=1)]),
    (forward, "ALIGN", [dict(x=A + 2), dict(y=A + 2), dict(w=A + 2), dict(b=A + 1), dict(mean=A + 2), dict(rstd=A + 2), dict(codes=A + 8)]),
    (forward, "TOO_LARGE", [dict(cols=16385, ldx=16385, ldy=16385, ldc=16416, lds=513), dict(rows=BIG)]),
    (backward, "INVALID", [dict(kind=2), dict(dtype=2), dict(pdtype=2), dict(fmt=3), dict(gy=0), dict(gx=0), dict(fmt=0, x=0, ldx=40),
                           dict(fmt=0, x=A, ldx=39), dict(mean=0), dict(rstd=0), dict(kind=1), dict(gw=0), dict(codes=0)]),
    (backward, "ALIGN", [dict(gy=A + 2), dict(gx=A + 2), dict(w=A + 2), dict(gw=A + 2), dict(gb=A + 2), dict(ws=A + 8), dict(rstd=A + 2)]),
    (backward, "TOO_LARGE", [dict(cols=16385, ldg=16385, ldgx=16385, ldc=16416, lds=513)]),
]


@pytest.mark.parametrize("call,status,changes", REFUSED, ids=["%s-%s" % (c.__name__, s) for c, s, _ in REFUSED])
def test_refusals(ampq, call, status, changes):
    for change in changes:
        assert call(ampq.lib(), **change) == getattr(ampq, "ERR_" + status), change


def test_workspace_queries_refuse(ampq):
    L, n = ampq.lib(), C.c_longlong()
    assert L.ampq_norm_backward_workspace(0, 4, 4, None) == ampq.ERR_INVALID
    assert L.ampq_norm_backward_workspace(0, -1, 4, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_norm_backward_workspace(0, 4, 16385, C.byref(n)) == ampq.ERR_TOO_LARGE
    assert L.ampq_ckpt_weight_grad_workspace(0, 0, None, 4, 1, 1, 4, 4, None) == ampq.ERR_INVALID
    assert L.ampq_ckpt_weight_grad_workspace(0, 7, None, 4, 1, 1, 4, 4, C.byref(n)) == ampq.ERR_INVALID
    assert L.ampq_ckpt_weight_grad_workspace(0, 0, None, 4, 1 << 20, 1 << 20, 4, 4, C.byref(n)) == ampq.ERR_TOO_LARGE


def test_no_device_is_an_error(ampq):
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    L, n = ampq.lib(), C.c_longlong()
    assert pack(L) == unpack(L) == wgrad(L) == forward(L) == backward(L) == ampq.ERR_CUDA
    assert L.ampq_norm_backward_workspace(0, 4, 4, C.byref(n)) == ampq.ERR_CUDA


def test_tensors_are_checked(ampq):
    from paper_2505_13060_b200 import checkpoint as ckpt

    x = torch.zeros(4, 40)
    for call in (lambda: ckpt.pack(x), lambda: ckpt.norm_forward(x, None, None, 1e-5)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    with pytest.raises(ValueError):
        ckpt.Packed(codes, scales, 40, 1)
    with pytest.raises(TypeError):
        ckpt.Packed(codes.float(), scales, 40, 1)


@pytest.mark.parametrize("fmt", [1, 2])
def test_reference_properties(fmt):
    """The reference itself: the relative error of a stored value is at most half a step of the format, every decoded value
    is a bf16 number and is stored as itself, and no smaller power of two would hold the group."""
    rng = np.random.default_rng(fmt)
    mant, bias, fmax, top = ref.FORMATS[fmt]
    x = rng.standard_normal((200, 70)) * 10.0 ** rng.integers(-20, 20, (200, 1))
    x = x.astype(np.float32).astype(np.float64)
    codes, scales = ref.pack(x, fmt)
    v = ref.unpack(codes, scales, 70, fmt)
    p = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)[:, :70]
    normal = np.abs(x) >= 2.0 ** (1 - bias) * p
    assert (np.abs(v - x)[normal] <= 2.0 ** -(mant + 1) * np.abs(x)[normal]).all()
    assert (np.abs(v - x) <= np.maximum(2.0 ** -(mant + 1) * np.abs(x), 2.0 ** (-bias - mant) * p)).all()
    assert np.array_equal(torch.tensor(v).bfloat16().double().numpy(), v)
    # stored again, a value stays itself (the scale may be another one: the group's maximum was rounded)
    codes2, scales2 = ref.pack(v, fmt)
    assert np.array_equal(ref.unpack(codes2, scales2, 70, fmt), v)
    a = np.abs(np.pad(x, ((0, 0), (0, 26)))).reshape(200, 3, 32).max(2)
    assert (fmax * 2.0 ** (scales.astype(float) - 127) >= a).all() and (fmax * 2.0 ** (scales.astype(float) - 128) < a).all()


def test_calibrator_refuses_unknown_checkpoints():
    from paper_2505_13060_b200 import hooks

    with pytest.raises(ValueError, match="checkpoint"):
        hooks.Calibrator(None, torch.nn.Linear(2, 2), 1, checkpoint=3)
