"""What is measured of the operators around a decoder's linear layers and norms.

A calibration (or training) step of a decoder runs, besides its linear layers and the norms of whole rows, three more
operators: the embedding lookup in front (``embed``, gradient ``embed_grad``), the norms of queries and keys for each
head with the position rotation (``heads``, ``heads_grad``), and the loss behind the head, here the divergence from a
teacher of which only the top logits of each token are known (``distill``, ``distill_grad``).

Formulas:

  heads:   r = 1 / sqrt(mean_c x^2 + eps), n = x * r * w for each head of each token; then, with the table's angle of
           the token's position, pairs of columns i, j are rotated: y_i = n_i cos - n_j sin, y_j = n_j cos + n_i sin.
           Pairs of the first `rot` columns are (i, i + rot/2) or, interleaved, (2i, 2i + 1); the rest stays as it is.
           With a format the input's 8-bit checkpoint is written too: groups of 32 columns of a head, a power-of-two scale
  heads_grad:  t = the gradient rotated back, h = x * r, u = t * w:  gx = r * (u - h * mean_c(u * h)),  gw = sum t * h
           over tokens and heads
  embed:   y[n] = scale * W[token[n]]
  embed_grad:  gW[v] = scale * sum of gy[n] over the n with token[n] = v; 0 for the padding token and for unused rows
  distill: entries k with index >= 0; p = softmax of the teacher's logits / T over a row's entries, q = softmax of
           the student's logits / T over all columns; loss = T^2 * sum_k p_k * (log p_k - log q[index_k]).  What the
           backward pass needs besides: the largest logit and sum_j exp((s_j - largest) / T).  Rows without an
           entry (prompt tokens, padding) have loss 0, statistics 0 and gradient 0
  distill_grad:  gs_j = gl * T * (q_j - sum of p_k over the k with index_k = j)
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


def _heads(op, dtype, fmt, batch, tokens, hq, hk, d, rot, interleaved=False, fused=False):
    return {"op": op, "dtype": dtype, "fmt": fmt, "batch": batch, "tokens": tokens, "hq": hq, "hk": hk, "d": d, "rot": rot,
            "interleaved": interleaved, "fused": fused}


def _embed(op, dtype, tokens, vocab, cols, padding=False):
    return {"op": op, "dtype": dtype, "tokens": tokens, "vocab": vocab, "cols": cols, "padding": padding}


def _distill(op, dtype, rows, vocab, top, temperature=1.0, unused=0, ragged=False, masked=0):
    return {"op": op, "dtype": dtype, "rows": rows, "vocab": vocab, "top": top, "temperature": temperature, "unused": unused,
            "ragged": ragged, "masked": masked}


def listed():
    return [
        # eight sequences that are each given their next token, far into a long context: latency
        {"name": "heads-next-token"} | _heads("heads", "bf16", "none", 8, 1, 32, 32, 128, 128),
        # a 70B-shaped block's fused projection, 2 samples of 4096 tokens, its q and k read in place and kept in 8 bits
        {"name": "heads-70b"} | _heads("heads", "bf16", "e4m3", 2, 4096, 64, 8, 128, 128, fused=True),
        # a ragged batch in fp32, heads of 80 columns of which the first half is rotated
        {"name": "heads-grad-odd"} | _heads("heads_grad", "f32", "none", 3, 331, 12, 12, 80, 40, interleaved=True),
        # the 70B-shaped block's backward pass from 8 bits
        {"name": "heads-grad-70b"} | _heads("heads_grad", "bf16", "e4m3", 2, 4096, 64, 8, 128, 128),
        # the next tokens of eight sequences
        {"name": "embed-next-token"} | _embed("embed", "bf16", 8, 32000, 4096),
        # 2 samples of 4096 tokens of a 70B-shaped model
        {"name": "embed-70b"} | _embed("embed", "bf16", 8192, 128000, 8192),
        # a toy model of odd sizes whose batch is padded
        {"name": "embed-grad-odd"} | _embed("embed_grad", "f32", 1000, 5003, 257, padding=True),
        # a 70B-shaped model's table: most of its rows are used by no token
        {"name": "embed-grad-70b"} | _embed("embed_grad", "bf16", 8192, 128000, 8192),
        # a toy vocabulary: latency
        {"name": "distill-toy"} | _distill("distill", "f32", 128, 1009, 8),
        # a 70B-shaped head on a sample of 4096 tokens, some of them of the prompt
        {"name": "distill-70b"} | _distill("distill", "bf16", 4096, 128000, 64, unused=20),
        # rows at no vector's border, short lists, a vocabulary with masked columns, soft targets
        {"name": "distill-grad-odd"} | _distill("distill_grad", "bf16", 1021, 50021, 100, 2.0, ragged=True, masked=21),
        # the 70B-shaped head's backward pass
        {"name": "distill-grad-70b"} | _distill("distill_grad", "bf16", 4096, 128000, 64, unused=20),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; half of the larger ones are multiples of 64."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    if n > 64 and rng.random() < 0.5:
        n -= n % 64
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["heads", "heads_grad", "embed", "embed_grad", "distill", "distill_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("heads", "heads_grad"):
        d = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 160, 256, 2 * rng.randint(1, 128)])
        rot = rng.choice([d, d, d // 4 * 2])
        hk = _spread(rng, 1, 16)
        hq = hk * rng.choice([1, 2, 4])
        batch = rng.choice([1, 1, 2, 3, 8])
        tokens = _spread(rng, 1, max(1, min(4096, 8192 * 72 * 128 * 2 // (BYTES[dtype] * batch * (hq + hk) * d))))
        return _heads(op, dtype, rng.choice(["none", "e4m3", "e5m2"]), batch, tokens, hq, hk, d, rot, rng.random() < 0.3, rng.random() < 0.5)
    if op in ("embed", "embed_grad"):
        cols = _spread(rng, 1, 8192)
        return _embed(op, dtype, _spread(rng, 1, 8192), _spread(rng, 1, 128000 if dtype == "bf16" else 64000), cols, rng.random() < 0.3)
    vocab = _spread(rng, 16, 128000)
    rows = _spread(rng, 1, 4096 if dtype == "bf16" else 2048)
    return _distill(op, dtype, rows, vocab, _spread(rng, 1, min(vocab, 256)), rng.choice([1.0, 1.0, 2.0, 0.7]), rng.choice([0, 0, 20, 2]),
                    rng.random() < 0.4, rng.choice([0, 0, vocab // 10]))


# -- inputs -----------------------------------------------------------------------------------------------------


def _power(e):
    """2^e in fp32, from its bits: exact for whole e of [-126, 127]."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _power64(e):
    """2^e in fp64, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _prepare_heads(case, s, g):
    dtype, d, rot = DTYPE[case["dtype"]], case["d"], case["rot"]
    batch, tokens = case["batch"], case["tokens"]
    total = (case["hq"] + 2 * case["hk"]) * d
    # N(0, 1), one channel in a hundred (at least one) twenty times as large
    factor = torch.ones(total, device="cuda")
    factor[torch.randperm(total, device="cuda", generator=g)[: max(1, total // 100)]] = 20.0
    qkv = torch.randn(batch, tokens, total, device="cuda", generator=g).mul_(factor).to(dtype)
    q, k = qkv[..., : case["hq"] * d], qkv[..., case["hq"] * d : (case["hq"] + case["hk"]) * d]
    if not case["fused"]:
        q, k = q.contiguous(), k.contiguous()
    s["q"], s["k"] = q.unflatten(-1, (case["hq"], d)), k.unflatten(-1, (case["hk"], d))
    for name in ("wq", "wk"):
        s[name] = (1.0 + 0.1 * torch.randn(d, device="cuda", generator=g)).to(dtype)
    # the model's table of angles; every sequence begins somewhere in a context of 32768
    length = 32768
    freq = 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / max(rot, 1))
    angle = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    start = torch.randint(0, length - tokens + 1, (batch, 1), device="cuda", generator=g)
    s["positions"] = start + torch.arange(tokens, device="cuda")
    if case["op"] == "heads":
        return
    for name, heads in (("q", case["hq"]), ("k", case["hk"])):
        x = s[name]
        s["r" + name] = (x.double().square().mean(-1) + EPS).rsqrt().float()
        if case["fmt"] != "none":
            x2 = x.reshape(-1, d)
            values, scales = _pack_plain(x2, case["fmt"])
            codes = torch.zeros(x2.shape[0], scales.shape[1] * GROUP, device="cuda", dtype=torch.uint8)
            codes[:, :d] = values.view(torch.uint8)
            s[name] = (codes, scales)
        s["g" + name] = torch.randn(batch, tokens, heads, d, device="cuda", generator=g).mul_(1e-3).to(dtype)


def _prepare_embed(case, s, g):
    dtype, vocab, n, cols = DTYPE[case["dtype"]], case["vocab"], case["tokens"], case["cols"]
    s["scale"] = float(cols) ** 0.5
    # frequent tokens first, as vocabularies are sorted; where the batch is padded its last third is token 0
    u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
    tokens = (torch.exp(u * np.log(vocab + 1.0)) - 1).long().clamp(max=vocab - 1)
    if case["padding"]:
        tokens[n - n // 3 :] = 0
    s["tokens"] = tokens
    if case["op"] == "embed":
        s["weight"] = torch.randn(vocab, cols, device="cuda", generator=g).mul_(0.02).to(dtype)
    else:
        s["gy"] = torch.randn(n, cols, device="cuda", generator=g).mul_(1e-4).to(dtype)


def _prepare_distill(case, s, g):
    dtype, rows, vocab, top, T = DTYPE[case["dtype"]], case["rows"], case["vocab"], case["top"], case["temperature"]
    logits = torch.randn(rows, vocab, device="cuda", generator=g).mul_(2.5)
    if case["masked"]:
        logits[:, vocab - case["masked"] :] = float("-inf")
    # the teacher's largest logits; the student is near the teacher where that is sure
    kept = min(top, vocab - case["masked"])
    value, index = logits.topk(kept, dim=1)
    teacher = torch.full((rows, top), 0.0, device="cuda")
    indices = torch.full((rows, top), -1, device="cuda")
    teacher[:, :kept], indices[:, :kept] = value + 1.5 * torch.randn(rows, kept, device="cuda", generator=g), index
    if case["ragged"]:
        length = torch.randint(1, top + 1, (rows, 1), device="cuda", generator=g)
        indices[torch.arange(top, device="cuda") >= length] = -1
    if case["unused"]:
        indices[case["unused"] - 1 :: case["unused"]] = -1
    s["logits"], s["indices"], s["teacher"] = logits.to(dtype), indices, teacher
    if case["op"] == "distill":
        return
    # what the forward pass left, and the gradient of a mean over tokens of different weight
    s["stats"] = torch.empty(rows, 2, device="cuda")
    for at in range(0, rows, 512):
        x = s["logits"][at : at + 512].float()
        largest = x.amax(1, keepdim=True)
        s["stats"][at : at + 512] = torch.cat([largest, ((x - largest) / T).exp().sum(1, keepdim=True)], 1)
    s["stats"][(indices < 0).all(1)] = 0.0
    s["gl"] = (0.5 + torch.rand(rows, device="cuda", generator=g)) / rows


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case, seed=seed)
    kind = case["op"].removesuffix("_grad")
    {"heads": _prepare_heads, "embed": _prepare_embed, "distill": _prepare_distill}[kind](case, s, g)
    return s


# -- the plain form ---------------------------------------------------------------------------------------------


def _pack_plain(x, fmt):
    """(values the codes stand for, in the format's own type; scale bytes) of x [rows, cols]."""
    mant, emin, fmax, top, kind, _ = FORMAT[fmt]
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    v = torch.nn.functional.pad(x.float(), (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    a = v.abs().amax(2)
    m, k = torch.frexp(a)  # a = m * 2^k, fmax = mf * 2^kf, both m in [0.5, 1)
    mf, kf = np.frexp(fmax)
    e = k - int(kf) + (m > float(mf)).int()
    e = torch.where(a == 0, torch.zeros_like(e), e.clamp(-110, top))
    y = (v * _power(-e)[..., None]).clamp(-fmax, fmax)
    _, ey = torch.frexp(y)
    step = _power((ey - 1).clamp(min=emin) - mant)
    q = torch.copysign(torch.round(y / step) * step, y).clamp(-fmax, fmax)
    return q.view(rows, groups * GROUP)[:, :cols].to(kind), (e + 127).to(torch.uint8)


def _unpack_plain(codes, scales, cols, fmt):
    """fp32 values of a checkpoint."""
    v = codes.view(FORMAT[fmt][4]).float().view(codes.shape[0], -1, GROUP)
    return (v * _power(scales.int() - 127)[..., None]).view(codes.shape[0], -1)[:, :cols]


def _rotate(n, cos, sin, rot, interleaved):
    """The first `rot` columns of n [batch, tokens, heads, d] rotated by angles [batch, tokens, rot / 2]."""
    cos, sin = cos[:, :, None, :], sin[:, :, None, :]
    a, b = (n[..., 0:rot:2], n[..., 1:rot:2]) if interleaved else (n[..., : rot // 2], n[..., rot // 2 : rot])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([ya, yb], -1).flatten(-2) if interleaved else torch.cat([ya, yb], -1)
    return torch.cat([both, n[..., rot:]], -1)


def _heads_plain(s):
    cos, sin = s["cos"][s["positions"]], s["sin"][s["positions"]]
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        rstd = (x.square().mean(-1) + EPS).rsqrt()
        n = x * rstd[..., None] * s["w" + name].float()
        out["y" + name] = _rotate(n, cos, sin, s["rot"], s["interleaved"]).to(s[name].dtype)
        out["r" + name] = rstd
        if s["fmt"] != "none":
            out["values_" + name], out["scales_" + name] = _pack_plain(s[name].reshape(-1, s["d"]), s["fmt"])
    return out


def _heads_grad_plain(s):
    cos, sin = s["cos"][s["positions"]], s["sin"][s["positions"]]
    out = {}
    for name in ("q", "k"):
        gy, w, rstd = s["g" + name], s["w" + name], s["r" + name][..., None]
        x = s[name].float() if s["fmt"] == "none" else _unpack_plain(*s[name], s["d"], s["fmt"]).view(gy.shape)
        t = _rotate(gy.float(), cos, -sin, s["rot"], s["interleaved"])
        h = x * rstd
        u = t * w.float()
        out["gx" + name] = (rstd * (u - h * (u * h).mean(-1, keepdim=True))).to(gy.dtype)
        out["gw" + name] = (t * h).sum((0, 1, 2)).to(w.dtype)
    return out


def _embed_plain(s):
    return {"y": (s["weight"][s["tokens"]].float() * s["scale"]).to(s["weight"].dtype)}


def _embed_grad_plain(s):
    total = torch.zeros(s["vocab"], s["cols"], device="cuda")
    total.index_add_(0, s["tokens"], s["gy"].float())
    if s["padding"]:
        total[0] = 0.0
    return {"gw": (total * s["scale"]).to(s["gy"].dtype)}


def _targets_plain(s):
    """The teacher's probabilities of the entries (0 where there is none), and which entries there are."""
    there = s["indices"] >= 0
    t = torch.where(there, s["teacher"].float() / s["temperature"], torch.full_like(s["teacher"], float("-inf"), dtype=torch.float32))
    some = there.any(1, keepdim=True)
    t = torch.where(some, t - t.amax(1, keepdim=True), torch.zeros_like(t))
    e = torch.where(there, t.exp(), torch.zeros_like(t))
    p = e / torch.where(some, e.sum(1, keepdim=True), torch.ones_like(t[:, :1]))
    return p, there, some


def _distill_plain(s):
    T = s["temperature"]
    p, there, some = _targets_plain(s)
    x = s["logits"].float()
    largest = x.amax(1, keepdim=True)
    total = ((x - largest) / T).exp().sum(1, keepdim=True)
    log_q = (x.gather(1, s["indices"].clamp(min=0)) - largest) / T - total.log()
    terms = p * (torch.where(p > 0, p, torch.ones_like(p)).log() - log_q)
    loss = T * T * torch.where(there & (p > 0), terms, torch.zeros_like(terms)).sum(1)
    stats = torch.cat([largest, total], 1)
    return {"loss": torch.where(some[:, 0], loss, torch.zeros_like(loss)), "stats": torch.where(some, stats, torch.zeros_like(stats))}


def _distill_grad_plain(s):
    T = s["temperature"]
    p, there, some = _targets_plain(s)
    largest, total = s["stats"][:, :1], s["stats"][:, 1:]
    q = ((s["logits"].float() - largest) / T).exp() / total
    q.scatter_add_(1, s["indices"].clamp(min=0), -p)
    g = q * (s["gl"] * T)[:, None]
    return {"gs": torch.where(some, g, torch.zeros_like(g)).to(s["logits"].dtype)}


# -- the framework's operators ------------------------------------------------------------------------------------


def _run_own(s):
    from paper_2505_13060_b200 import binding, checkpoint, decoder

    op = s["op"]
    if op == "embed":
        return {"y": decoder.embed(s["tokens"], s["weight"], s["scale"])}
    if op == "embed_grad":
        return {"gw": decoder.embed_backward(s["tokens"], s["gy"], s["vocab"], s["scale"], padding_idx=0 if s["padding"] else None)}
    if op == "distill":
        loss, stats = decoder.distill_forward(s["logits"], s["indices"], s["teacher"], s["temperature"])
        return {"loss": loss, "stats": stats}
    if op == "distill_grad":
        return {"gs": decoder.distill_backward(s["gl"], s["logits"], s["indices"], s["teacher"], s["stats"], s["temperature"])}
    fmt = FORMAT[s["fmt"]][5] if s["fmt"] != "none" else binding.FMT_BASE
    rotation = (s["cos"], s["sin"], s["positions"])
    if op == "heads":
        yq, yk, rq, rk, pq, pk = decoder.head_norm_forward(s["q"], s["k"], s["wq"], s["wk"], *rotation, EPS, s["interleaved"], fmt)
        out = {"yq": yq, "rq": rq, "yk": yk, "rk": rk}
        if fmt != binding.FMT_BASE:
            for name, p in (("q", pq), ("k", pk)):
                out |= {"values_" + name: p.codes.view(FORMAT[s["fmt"]][4])[:, : s["d"]], "scales_" + name: p.scales}
        return out
    xq, xk = (s[name] if s["fmt"] == "none" else checkpoint.Packed(*s[name], s["d"], fmt) for name in ("q", "k"))
    gxq, gxk, gwq, gwk = decoder.head_norm_backward(s["gq"], s["gk"], xq, xk, s["rq"], s["rk"], s["wq"], s["wk"], *rotation, s["interleaved"])
    return {"gxq": gxq, "gwq": gwq, "gxk": gxk, "gwk": gwk}


def run(state):
    if own:
        return _run_own(state)
    plain = {"heads": _heads_plain, "heads_grad": _heads_grad_plain, "embed": _embed_plain, "embed_grad": _embed_grad_plain,
             "distill": _distill_plain, "distill_grad": _distill_grad_plain}
    return plain[state["op"]](state)


def work(case):
    b, op = BYTES[case["dtype"]], case["op"]
    if op in ("heads", "heads_grad"):
        heads = case["batch"] * case["tokens"] * (case["hq"] + case["hk"])
        n = heads * case["d"]
        kept = heads * (case["d"] + -(-case["d"] // GROUP)) if case["fmt"] != "none" else 0
        angles = case["batch"] * case["tokens"] * (4 * case["rot"] + 8)
        if op == "heads":
            return {"bytes": 2 * b * n + kept + 4 * heads + angles, "flops": 8 * n}
        return {"bytes": 2 * b * n + (kept or b * n) + 4 * heads + angles, "flops": 16 * n}
    if op in ("embed", "embed_grad"):
        n, vocab, cols = case["tokens"], case["vocab"], case["cols"]
        if op == "embed":  # a row that several tokens share is read once: the expected number of different tokens
            share = np.diff(np.log(np.arange(1, vocab + 2))) / np.log(vocab + 1.0)
            rows = int(round(float((1.0 - (1.0 - share) ** n).sum())))
            return {"bytes": b * (n + rows) * cols + 8 * n, "flops": n * cols}
        used = n - (n // 3 if case["padding"] else 0)
        return {"bytes": b * (used + vocab) * cols + 8 * n, "flops": (used + vocab) * cols}
    rows = case["rows"] - (case["rows"] // case["unused"] if case["unused"] else 0)
    lists = 12 * case["rows"] * case["top"]
    if op == "distill":
        return {"bytes": b * rows * case["vocab"] + lists + 12 * case["rows"], "flops": 4 * rows * case["vocab"]}
    return {"bytes": b * (rows + case["rows"]) * case["vocab"] + lists + 12 * case["rows"], "flops": 5 * rows * case["vocab"]}


# -- the definition in 64 bits --------------------------------------------------------------------------------------


def _grid(fmt):
    """Every value >= 0 of the format, ascending: value i has code i."""
    mant, emin, top = FORMAT[fmt][:3]
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
    values = []
    for block in x.split(1 << 16):
        v = torch.nn.functional.pad(block.double(), (0, -block.shape[1] % GROUP)).reshape(-1, GROUP)
        a = v.abs().max(1).values
        p = torch.where(a > 0, powers[torch.searchsorted(powers * grid[-1], a).clamp(max=powers.numel() - 1)], torch.ones_like(a))
        y = v.abs() / p[:, None]
        lo = torch.searchsorted(between, y)  # the middle points below y
        tie = (lo < between.numel()) & (between[lo.clamp(max=between.numel() - 1)] == y)
        code = torch.where(tie, lo + (lo & 1), lo)  # at a middle point the even one of the two codes
        values.append((grid[code] * torch.sign(v)).reshape(block.shape[0], -1)[:, : x.shape[1]])
    return torch.cat(values)


def _exact_kept(codes, scales, d, fmt):
    """A checkpoint's values in 64 bits, by the list of all values."""
    grid = _grid(fmt)
    c = codes.long()
    v = torch.where(c >= 128, -grid[(c & 127).clamp(max=grid.numel() - 1)], grid[c.clamp(max=grid.numel() - 1)])
    return (v * _power64(scales.int() - 127).repeat_interleave(GROUP, 1))[:, :d]


def _exact_heads(case, s):
    """The rotation as the multiplication of each pair, as a complex number, by the angle's."""
    rot, d, grad = case["rot"], case["d"], case["op"] == "heads_grad"
    angle = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]][:, :, None, :]
    columns = torch.arange(rot, device="cuda")
    first, second = (columns[0::2], columns[1::2]) if case["interleaved"] else (columns[: rot // 2], columns[rot // 2 :])

    def turned(x, by):
        y = x.clone()
        z = torch.complex(x[..., first], x[..., second]) * by
        y[..., first], y[..., second] = z.real, z.imag
        return y

    out = {}
    for name in ("q", "k"):
        w = s["w" + name].double()
        if not grad:
            x = s[name].double()
            r = 1.0 / torch.sqrt(torch.einsum("bthc,bthc->bth", x, x) / d + EPS)
            out["y" + name], out["r" + name] = turned(torch.einsum("bthc,bth,c->bthc", x, r, w), angle), r
            if case["fmt"] != "none":
                out |= {"values_" + name: _exact_pack(s[name].reshape(-1, d), case["fmt"]), "scales_" + name: None}
            continue
        gy, r = s["g" + name].double(), s["r" + name].double()
        x = s[name].double() if case["fmt"] == "none" else _exact_kept(*s[name], d, case["fmt"]).reshape(gy.shape)
        t = turned(gy, angle.conj())
        h = torch.einsum("bthc,bth->bthc", x, r)
        mean = torch.einsum("bthc,bthc,c->bth", t, h, w) / d
        out["gx" + name] = torch.einsum("bthc,bth->bthc", t * w - h * mean[..., None], r)
        out["gw" + name] = torch.einsum("bthc,bthc->c", t, h)
    return out


def _exact_embed(case, s):
    if case["op"] == "embed":
        return {"y": torch.nn.functional.embedding(s["tokens"], s["weight"]).double() * s["scale"]}
    order = torch.argsort(s["tokens"], stable=True)
    token = s["tokens"][order]
    gw = torch.zeros(case["vocab"], case["cols"], device="cuda", dtype=torch.float64)
    used, count = torch.unique_consecutive(token, return_counts=True)
    ends = count.cumsum(0)
    for at in range(0, case["cols"], 512):  # differences of running sums: 64 bits leave 32 whole
        run = torch.nn.functional.pad(s["gy"][order, at : at + 512].double().cumsum(0), (0, 0, 1, 0))
        gw[used, at : at + 512] = (run[ends] - run[ends - count]) * s["scale"]
    if case["padding"]:
        gw[0] = 0.0
    return {"gw": gw}


def _exact_distill(case, s):
    T, rows, vocab = case["temperature"], case["rows"], case["vocab"]
    grad = case["op"] == "distill_grad"
    out = {"gs": torch.zeros(rows, vocab, device="cuda", dtype=torch.float64)} if grad else {
        "loss": torch.zeros(rows, device="cuda", dtype=torch.float64), "stats": torch.zeros(rows, 2, device="cuda", dtype=torch.float64)}
    for at in range(0, rows, 256):
        some = torch.arange(at, min(at + 256, rows), device="cuda")
        some = some[(s["indices"][some] >= 0).any(1)]
        if not some.numel():
            continue
        index, there = s["indices"][some].clamp(min=0), s["indices"][some] >= 0
        log_p = torch.log_softmax((s["teacher"][some].double() / T).masked_fill(~there, float("-inf")), 1)
        x = s["logits"][some].double()
        if grad:
            q = torch.exp((x - s["stats"][some, :1].double()) / T) / s["stats"][some, 1:].double()
            target = torch.zeros_like(q).scatter_add_(1, index, log_p.exp())
            out["gs"][some] = (q - target) * (s["gl"][some].double() * T)[:, None]
        else:
            log_q = torch.log_softmax(x / T, 1).gather(1, index)
            out["loss"][some] = T * T * (log_p.exp() * (log_p - log_q)).masked_fill(~there | (log_p.exp() == 0), 0.0).sum(1)
            largest = x.max(1, keepdim=True).values
            out["stats"][some] = torch.cat([largest, torch.exp((x - largest) / T).sum(1, keepdim=True)], 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["op"].removesuffix("_grad")
    return {"heads": _exact_heads, "embed": _exact_embed, "distill": _exact_distill}[kind](case, s)
