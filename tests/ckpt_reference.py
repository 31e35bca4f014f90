"""8-bit checkpoints and norms from their definitions, in 64 bits on the host.
Shares nothing with the library: the FP8 values come from the format's
definition, scales and codes from searches in lists of them."""
import numpy as np

GROUP = 32
#: format number: (mantissa bits, exponent bias, largest finite value, largest scale exponent)
FORMATS = {1: (3, 7, 448.0, 119), 2: (2, 15, 57344.0, 112)}


def grid(fmt):
    """Values of the codes 0, 1, ... up to the largest finite one."""
    mant, bias, fmax, _ = FORMATS[fmt]
    out, code = [], 0
    while not out or out[-1] < fmax:
        field, frac = code >> mant, code & ((1 << mant) - 1)
        out.append(frac * 2.0 ** (1 - bias - mant) if field == 0 else (1 + frac / (1 << mant)) * 2.0 ** (field - bias))
        code += 1
    return np.array(out)


def pack(x, fmt):
    """x [rows, cols] in float64 -> (codes [rows, groups * 32], scales [rows, groups])."""
    g = grid(fmt)
    mid = (g[1:] + g[:-1]) / 2
    top = FORMATS[fmt][3]
    exps = np.arange(-110, top + 1)
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    v = np.zeros((rows, groups * GROUP))
    v[:, :cols] = x
    v = v.reshape(rows, groups, GROUP)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[..., None], 0.0, v)
    a = np.abs(v).max(2)
    at = np.minimum(np.searchsorted(g[-1] * 2.0 ** exps, a), len(exps) - 1)
    e = np.where(a > 0, exps[at], 0)
    y = np.abs(v) * 2.0 ** -e[..., None].astype(np.float64)
    lo = np.searchsorted(mid, y)
    tie = (lo < len(mid)) & (mid[np.minimum(lo, len(mid) - 1)] == y)
    code = np.where(tie & (lo % 2 == 1), lo + 1, lo)
    code = np.where(np.signbit(v), code | 128, code)
    code = np.where(bad[..., None], 0, code)
    scales = np.where(bad, 255, e + 127)
    return code.reshape(rows, -1).astype(np.uint8), scales.astype(np.uint8)


def unpack(codes, scales, cols, fmt):
    g = grid(fmt)
    c = codes.astype(np.int64)
    v = np.where(c >= 128, -1.0, 1.0) * g[np.minimum(c & 127, len(g) - 1)]
    p = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(p, GROUP, axis=1))[:, :cols]
