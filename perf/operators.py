"""What is measured of the 8-bit activation checkpoints and the norms.

A calibration (or training) step keeps the inputs of its linear layers and norms from the forward pass for the
backward pass.  Kept in 8 bits with one power-of-two scale per group of 32 columns they take half the memory of
bf16.  Five operators: write a checkpoint (``pack``), read it (``unpack``), form a linear layer's weight gradient
from it sample by sample (``wgrad``), and the norms' forward pass (``norm``), which writes the checkpoint of its
input on the way, and backward pass (``norm_grad``), which reads it.

Formulas, for a row group x of at most 32 consecutive columns and a format with largest finite value fmax:

  a = max|x|, e = the smallest integer with fmax * 2^e >= a, within [-110, 119] (E4M3) or [-110, 112] (E5M2), 0 for a = 0
  code = x * 2^-e rounded to the nearest value of the format, ties to the even code, saturating; the scale byte is e + 127
  a group with an Inf or a NaN: scale byte 255, codes 0, decoded as NaN
  decoded value = code * 2^e

  wgrad:      gW[r] = gY[r]^T X^[r],  gb[r] = column sums of gY[r]
  layer norm: y = (x - mean) * rstd * w + b, rstd = 1 / sqrt(var + eps);  rms norm: y = x * rstd * w, rstd = 1 / sqrt(mean x^2 + eps)
  norm_grad:  h = (x - mean) * rstd, t = gy * w, gx = rstd * (t - mean(t) - h * mean(t * h)), gw = sum gy * h, gb = sum gy
              (rms norm: mean = 0, no mean(t) term, no gb)
"""
import numpy as np
import torch

own = False

GROUP = 32
EPS = 1e-5
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
#: format: (mantissa bits, smallest normal exponent, fmax, largest scale exponent, torch type, number in the library)
FORMAT = {
    "e4m3": (3, -6, 448.0, 119, torch.float8_e4m3fn, 1),
    "e5m2": (2, -14, 57344.0, 112, torch.float8_e5m2, 2),
}


def listed():
    return [
        # the toy MLP's input, 8 samples of 128 tokens: latency counts
        {"name": "pack-toy", "op": "pack", "dtype": "f32", "fmt": "e4m3", "rows": 1024, "cols": 256, "wide": False},
        # the input of a 70B-shaped down projection, 2 samples of 4096 tokens: the largest checkpoint of a block
        {"name": "pack-70b-down", "op": "pack", "dtype": "bf16", "fmt": "e4m3", "rows": 8192, "cols": 28672, "wide": False},
        # odd sizes: rows that start at no vector's border
        {"name": "unpack-odd", "op": "unpack", "dtype": "f32", "fmt": "e4m3", "rows": 1000, "cols": 1001, "wide": False},
        # a 70B-shaped hidden state handed to code that wants the tensor itself
        {"name": "unpack-70b", "op": "unpack", "dtype": "bf16", "fmt": "e5m2", "rows": 8192, "cols": 8192, "wide": False},
        # a norm of the toy width: latency
        {"name": "norm-toy", "op": "norm", "kind": "layer", "dtype": "f32", "fmt": "e4m3", "rows": 1024, "cols": 256, "wide": False},
        # the norm before a 70B-shaped block, its input checkpointed on the way
        {"name": "norm-70b", "op": "norm", "kind": "rms", "dtype": "bf16", "fmt": "e4m3", "rows": 8192, "cols": 8192, "wide": False},
        # a layer norm whose input was kept in full, ragged batch and odd width
        {"name": "norm-grad-odd", "op": "norm_grad", "kind": "layer", "dtype": "bf16", "fmt": "none", "rows": 2047, "cols": 4099, "wide": False},
        # the norm before a 70B-shaped block, backward from 8 bits
        {"name": "norm-grad-70b", "op": "norm_grad", "kind": "rms", "dtype": "bf16", "fmt": "e4m3", "rows": 8192, "cols": 8192, "wide": False},
        # one layer of the toy MLP, 8 per-sample gradients in fp32: latency
        {"name": "wgrad-toy", "op": "wgrad", "dtype": "f32", "fmt": "e4m3", "R": 8, "rows": 128, "cols": 256, "out": 256, "wide": False},
        # odd sizes, gradient rows at no vector's border
        {"name": "wgrad-odd", "op": "wgrad", "dtype": "bf16", "fmt": "e5m2", "R": 3, "rows": 997, "cols": 1031, "out": 4093, "wide": False},
        # a 7B-shaped attention projection, 4 samples of 2048 tokens
        {"name": "wgrad-7b", "op": "wgrad", "dtype": "bf16", "fmt": "e4m3", "R": 4, "rows": 2048, "cols": 4096, "out": 4096, "wide": False},
        # a 70B-shaped gate projection, 2 samples of 4096 tokens: the largest product of a block
        {"name": "wgrad-70b-gate", "op": "wgrad", "dtype": "bf16", "fmt": "e4m3", "R": 2, "rows": 4096, "cols": 8192, "out": 28672, "wide": False},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; half of the larger ones are multiples of 64."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    if n > 64 and rng.random() < 0.5:
        n -= n % 64
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["pack", "unpack", "norm", "norm_grad", "wgrad", "wgrad"])
    case = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16"]), "fmt": rng.choice(["e4m3", "e4m3", "e5m2"]), "wide": rng.random() < 0.3}
    if op in ("norm", "norm_grad"):
        case |= {"kind": rng.choice(["layer", "rms"]), "rows": _spread(rng, 1, 8192), "cols": _spread(rng, 1, 8192)}
        if rng.random() < 0.3:
            case["fmt"] = "none"  # the input is kept in full, or not at all
    elif op == "wgrad":
        case |= {"R": rng.choice([1, 1, 2, 3, 4, 8]), "rows": _spread(rng, 1, 4096), "cols": _spread(rng, 1, 11008), "out": _spread(rng, 1, 11008)}
    else:
        case |= {"rows": _spread(rng, 1, 8192), "cols": _spread(rng, 1, 28672)}
    return case


# -- inputs -----------------------------------------------------------------------------------------------------


def _power(e):
    """2^e in fp32, from its bits: exact for whole e of [-126, 127]."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _power64(e):
    """2^e in fp64, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _laid(t, wide):
    """t itself, or as the leading columns of wider rows, the way a part of a fused projection lies in memory."""
    if not wide:
        return t
    full = torch.zeros(t.shape[0], t.shape[1] + 72, device="cuda", dtype=t.dtype)
    full[:, : t.shape[1]] = t
    return full[:, : t.shape[1]]


def _gradients(g, dtype, wide, rows, cols):
    return _laid(torch.randn(rows, cols, device="cuda", generator=g).mul_(1e-4).to(dtype), wide)


def _activations(g, dtype, wide, rows, cols):
    """N(0, 1) with one input channel in a thousand (at least one) a hundred times as large."""
    factor = torch.ones(cols, device="cuda")
    factor[torch.randperm(cols, device="cuda", generator=g)[: max(1, cols // 1000)]] = 100.0
    return _laid(torch.randn(rows, cols, device="cuda", generator=g).mul_(factor).to(dtype), wide)


def _checkpoint(x, fmt):
    """The checkpoint a forward pass left: codes [rows, cols rounded up to whole groups] and scale bytes [rows, groups]."""
    values, scales = _pack_plain(x, fmt)
    codes = torch.zeros(x.shape[0], scales.shape[1] * GROUP, device="cuda", dtype=torch.uint8)
    codes[:, : x.shape[1]] = values.view(torch.uint8)
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, wide, op = DTYPE[case["dtype"]], case["wide"], case["op"]
    s = dict(case, seed=seed)
    if op == "wgrad":
        rows = case["R"] * case["rows"]
        s["codes"], s["scales"] = _checkpoint(_activations(g, dtype, False, rows, case["cols"]), case["fmt"])
        s["gy"] = _gradients(g, dtype, wide, rows, case["out"])
        return s
    x = _activations(g, dtype, wide and op != "unpack", case["rows"], case["cols"])
    if op == "unpack":
        s["codes"], s["scales"] = _checkpoint(x, case["fmt"])
        return s
    s["x"] = x
    if op == "pack":
        return s
    s["w"] = (1.0 + 0.1 * torch.randn(case["cols"], device="cuda", generator=g)).to(dtype)
    s["b"] = (0.1 * torch.randn(case["cols"], device="cuda", generator=g)).to(dtype) if case["kind"] == "layer" else None
    if op == "norm":
        return s
    # what the forward pass left: the statistics of the input, and the input or its checkpoint
    xd = x.double()
    mean = xd.mean(1) if case["kind"] == "layer" else torch.zeros(case["rows"], device="cuda", dtype=torch.float64)
    s["rstd"] = ((xd - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    s["mean"] = mean.float() if case["kind"] == "layer" else None
    del xd
    if case["fmt"] != "none":
        s["codes"], s["scales"] = _checkpoint(x, case["fmt"])
        s["x"] = None
    s["gy"] = _gradients(g, dtype, wide, case["rows"], case["cols"])
    return s


# -- the plain form ---------------------------------------------------------------------------------------------


def _pack_plain(x, fmt):
    """(values the codes stand for, in the format's own type; scale bytes) of x [rows, cols]."""
    mant, emin, fmax, top, kind, _ = FORMAT[fmt]
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    v = torch.nn.functional.pad(x.float(), (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    a = v.abs().amax(2)
    bad = ~torch.isfinite(a)
    m, k = torch.frexp(a)  # a = m * 2^k, fmax = mf * 2^kf, both m in [0.5, 1)
    mf, kf = np.frexp(fmax)
    e = k - int(kf) + (m > float(mf)).int()
    e = torch.where(a == 0, torch.zeros_like(e), e.clamp(-110, top))
    e = torch.where(bad, torch.zeros_like(e), e)
    y = torch.where(bad[..., None], torch.zeros_like(v), v * _power(-e)[..., None]).clamp(-fmax, fmax)
    _, ey = torch.frexp(y)
    step = _power((ey - 1).clamp(min=emin) - mant)
    q = torch.round(y / step) * step
    q = torch.copysign(q, y).clamp(-fmax, fmax)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return q.view(rows, groups * GROUP)[:, :cols].to(kind), scales


def _unpack_plain(codes, scales, cols, fmt):
    """fp32 values of a checkpoint."""
    v = codes.view(FORMAT[fmt][4]).float().view(codes.shape[0], -1, GROUP)
    p = torch.where(scales == 255, torch.full_like(v[..., 0], float("nan")), _power(scales.int().clamp(max=254) - 127))
    return (v * p[..., None]).view(codes.shape[0], -1)[:, :cols]


def _norm_plain(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True) if s["kind"] == "layer" else None
    c = x - mean if mean is not None else x
    rstd = (c.square().mean(1, keepdim=True) + EPS).rsqrt()
    y = c * rstd * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    out = {"y": y.to(s["x"].dtype), "rstd": rstd[:, 0]}
    if mean is not None:
        out["mean"] = mean[:, 0]
    if s["fmt"] != "none":
        out["values"], out["scales"] = _pack_plain(s["x"], s["fmt"])
    return out


def _norm_grad_plain(s):
    x = s["x"].float() if s["fmt"] == "none" else _unpack_plain(s["codes"], s["scales"], s["cols"], s["fmt"])
    gy, rstd = s["gy"].float(), s["rstd"][:, None]
    h = (x - s["mean"][:, None] if s["mean"] is not None else x) * rstd
    t = gy * s["w"].float()
    gx = t - h * (t * h).mean(1, keepdim=True)
    if s["mean"] is not None:
        gx = gx - t.mean(1, keepdim=True)
    out = {"gx": (gx * rstd).to(s["gy"].dtype), "gw": (gy * h).sum(0).to(s["w"].dtype)}
    if s["kind"] == "layer":
        out["gb"] = gy.sum(0).to(s["w"].dtype)
    return out


def _wgrad_plain(s):
    x = _unpack_plain(s["codes"], s["scales"], s["cols"], s["fmt"]).reshape(s["R"], s["rows"], s["cols"])
    gy = s["gy"].float().reshape(s["R"], s["rows"], s["out"])
    return {"gw": torch.matmul(gy.transpose(1, 2), x).to(s["gy"].dtype), "gb": gy.sum(1).to(s["gy"].dtype)}


# -- the framework's operators ------------------------------------------------------------------------------------


def _run_own(s):
    from paper_2505_13060_b200 import binding, checkpoint

    op, cols = s["op"], s["cols"]
    fmt = FORMAT[s["fmt"]][5] if s["fmt"] != "none" else binding.FMT_BASE
    if op == "pack":
        p = checkpoint.pack(s["x"], fmt)
        return {"values": p.codes.view(FORMAT[s["fmt"]][4])[:, :cols], "scales": p.scales}
    kept = checkpoint.Packed(s["codes"], s["scales"], cols, fmt) if "codes" in s else s.get("x")
    if op == "unpack":
        return {"x": checkpoint.unpack(kept, DTYPE[s["dtype"]])}
    if op == "wgrad":
        gw, gb = checkpoint.weight_grad(kept, s["gy"], samples=s["R"], bias=True)
        return {"gw": gw, "gb": gb}
    kind = binding.NORM_LAYER if s["kind"] == "layer" else binding.NORM_RMS
    if op == "norm":
        y, mean, rstd, p = checkpoint.norm_forward(s["x"], s["w"], s["b"], EPS, kind, fmt)
        out = {"y": y, "rstd": rstd}
        if mean is not None:
            out["mean"] = mean
        if p is not None:
            out |= {"values": p.codes.view(FORMAT[s["fmt"]][4])[:, :cols], "scales": p.scales}
        return out
    gx, gw, gb = checkpoint.norm_backward(s["gy"], kept, s["mean"], s["rstd"], s["w"], kind)
    return {"gx": gx, "gw": gw} | ({"gb": gb} if gb is not None else {})


def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "pack":
        values, scales = _pack_plain(state["x"], state["fmt"])
        return {"values": values, "scales": scales}
    if op == "unpack":
        return {"x": _unpack_plain(state["codes"], state["scales"], state["cols"], state["fmt"]).to(DTYPE[state["dtype"]])}
    return {"wgrad": _wgrad_plain, "norm": _norm_plain, "norm_grad": _norm_grad_plain}[op](state)


def work(case):
    b, n = BYTES[case["dtype"]], case["rows"] * case["cols"]
    kept = case["rows"] * (case["cols"] + -(-case["cols"] // GROUP)) if case["fmt"] != "none" else 0
    if case["op"] == "pack":
        return {"bytes": b * n + kept, "flops": 4 * n}
    if case["op"] == "unpack":
        return {"bytes": b * n + kept, "flops": n}
    if case["op"] == "norm":
        return {"bytes": 2 * b * n + kept, "flops": 8 * n}
    if case["op"] == "norm_grad":
        return {"bytes": 2 * b * n + (kept or b * n), "flops": 14 * n}
    R, N, C, K = case["R"], case["rows"], case["cols"], case["out"]
    return {"bytes": R * (b * N * K + kept + b * K * C), "flops": 2 * R * N * C * K + R * N * K}


# -- the definition in 64 bits --------------------------------------------------------------------------------------


def _grid(fmt):
    """Every value >= 0 of the format, ascending: value i has code i."""
    mant, emin = FORMAT[fmt][0], FORMAT[fmt][1]
    top = FORMAT[fmt][2]
    values, code = [], 0
    while not values or values[-1] < top:
        field, frac = code >> mant, code & ((1 << mant) - 1)
        values.append(frac * 2.0 ** (emin - mant) if field == 0 else (1 + frac / (1 << mant)) * 2.0 ** (field - 1 + emin))
        code += 1
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def _exact_pack(x, fmt):
    """Nearest value by search in the list of all values, ties to the even code; the scale exponent by search too."""
    top = FORMAT[fmt][3]
    grid = _grid(fmt)
    between = (grid[1:] + grid[:-1]) / 2
    powers = _power64(torch.arange(-110, top + 1, device="cuda"))
    reach = powers * grid[-1]
    values, scales = [], []
    for block in x.split(512):
        v = block.double()
        pad = -v.shape[1] % GROUP
        v = torch.cat([v, v.new_zeros(v.shape[0], pad)], 1).reshape(-1, GROUP)
        a = v.abs().max(1).values
        at = torch.searchsorted(reach, a).clamp(max=powers.numel() - 1)
        p = torch.where(a > 0, powers[at], torch.ones_like(a))
        y = v.abs() / p[:, None]
        lo = torch.searchsorted(between, y)  # the middle points below y
        tie = (lo < between.numel()) & (between[lo.clamp(max=between.numel() - 1)] == y)
        code = torch.where(tie, lo + (lo & 1), lo)  # at a middle point the even one of the two codes
        values.append((grid[code] * torch.sign(v)).reshape(block.shape[0], -1)[:, : x.shape[1]])
        scales.append(torch.where(a > 0, at - 110 + 127, torch.full_like(at, 127)).reshape(block.shape[0], -1))
    return torch.cat(values), torch.cat(scales)


def _exact_kept(s):
    """A checkpoint's values in 64 bits, by the list of all values."""
    grid = _grid(s["fmt"])
    c = s["codes"].long()
    v = torch.where(c >= 128, -grid[(c & 127).clamp(max=grid.numel() - 1)], grid[c.clamp(max=grid.numel() - 1)])
    p = _power64(s["scales"].int() - 127)
    return (v * p.repeat_interleave(GROUP, 1))[:, : s["cols"]]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        return {"values": _exact_pack(s["x"], s["fmt"])[0], "scales": None}
    if op == "unpack":
        return {"x": _exact_kept(s)}
    if op == "wgrad":
        x, gy = _exact_kept(s), s["gy"].double()
        N = case["rows"]
        gw = torch.stack([gy[r * N : (r + 1) * N].T @ x[r * N : (r + 1) * N] for r in range(case["R"])])
        return {"gw": gw, "gb": torch.stack([gy[r * N : (r + 1) * N].sum(0) for r in range(case["R"])])}
    n = float(case["cols"])
    if op == "norm":
        x = s["x"].double()
        mean = x.sum(1) / n if case["kind"] == "layer" else torch.zeros_like(x[:, 0])
        rstd = 1.0 / torch.sqrt((x - mean[:, None]).pow(2).sum(1) / n + EPS)
        y = torch.einsum("nc,n,c->nc", x - mean[:, None], rstd, s["w"].double())
        out = {"y": y if s["b"] is None else y + s["b"].double(), "rstd": rstd}
        if case["kind"] == "layer":
            out["mean"] = mean
        if case["fmt"] != "none":
            out |= {"values": _exact_pack(s["x"], s["fmt"])[0], "scales": None}
        return out
    x = s["x"].double() if case["fmt"] == "none" else _exact_kept(s)
    gy, w, rstd = s["gy"].double(), s["w"].double(), s["rstd"].double()
    layer = case["kind"] == "layer"
    h = torch.einsum("nc,n->nc", x - s["mean"].double()[:, None] if layer else x, rstd)
    both = torch.einsum("nc,nc,c->n", gy, h, w) / n
    only = (gy @ w) / n if layer else torch.zeros_like(both)
    gx = torch.einsum("n,nc->nc", rstd, gy * w - only[:, None] - h * both[:, None])
    out = {"gx": gx, "gw": torch.einsum("nc,nc->c", gy, h)}
    return out | ({"gb": gy.sum(0)} if layer else {})
