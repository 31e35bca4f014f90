"""The operators around a decoder's linear layers from their definitions, in 64 bits
on the host, each with the sizes that an error bound needs.  Shares nothing with the library."""
import numpy as np


def turn(x, cos, sin, rot, interleaved, back=False):
    """The first rot columns of x [..., heads, cols] turned by the angles [..., rot / 2] of each token; also the sums of the
    absolute values of the two products of each result."""
    cos, sin = cos[..., None, :], (-sin if back else sin)[..., None, :]
    y, size = x.copy(), np.abs(x)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    size[..., a] = np.abs(x[..., a] * cos) + np.abs(x[..., b] * sin)
    size[..., b] = np.abs(x[..., b] * cos) + np.abs(x[..., a] * sin)
    return y, size


def head_norm(x, w, cos, sin, rot, eps, interleaved):
    """x [batch, tokens, heads, cols]; cos and sin [batch, tokens, rot / 2].  (y, size of its terms, rstd)."""
    rstd = 1.0 / np.sqrt((x * x).mean(-1) + eps)
    n = x * rstd[..., None] * w
    return (*turn(n, cos, sin, rot, interleaved), rstd)


def head_norm_grad(gy, x, rstd, w, cos, sin, rot, interleaved):
    """(gx, gw, and what bounds their errors: size of u, size of the mean's terms, size of gw's terms)."""
    t, size = turn(gy, cos, sin, rot, interleaved, back=True)
    h = x * rstd[..., None]
    u = t * w
    gx = rstd[..., None] * (u - h * (u * h).mean(-1, keepdims=True))
    return gx, (t * h).sum((0, 1, 2)), size * np.abs(w), (size * np.abs(w * h)).mean(-1, keepdims=True) * np.abs(h), (size * np.abs(h)).sum((0, 1, 2))


def embed_grad(tokens, gy, vocab, scale, padding=None):
    """(gw, sums of absolute values, tokens of each row)."""
    gw, size, count = np.zeros((vocab, gy.shape[1])), np.zeros((vocab, gy.shape[1])), np.zeros(vocab)
    for n, t in enumerate(tokens):
        if 0 <= t < vocab and t != padding:
            gw[t] += gy[n]
            size[t] += np.abs(gy[n])
            count[t] += 1
    return gw * scale, size * abs(scale), count


def targets(indices, teacher, T):
    """Probabilities [rows, top] of the entries, 0 where there is none."""
    p = np.zeros(teacher.shape)
    for n in range(len(teacher)):
        there = indices[n] >= 0
        if there.any():
            e = np.exp((teacher[n, there] - teacher[n, there].max()) / T)
            p[n, there] = e / e.sum()
    return p


def distill(logits, indices, teacher, T):
    """Loss [rows] of finite lists and rows with a finite logit."""
    p = targets(indices, teacher, T)
    out = np.zeros(len(logits))
    for n in range(len(logits)):
        if not (indices[n] >= 0).any():
            continue
        m = logits[n].max()
        log_q = (logits[n] - m) / T - np.log(np.exp((logits[n] - m) / T).sum())
        for k, j in enumerate(indices[n]):
            if j >= 0 and p[n, k] > 0:
                out[n] += T * T * p[n, k] * (np.log(p[n, k]) - log_q[j])
    return out


def distill_grad(gl, logits, indices, teacher, T):
    """(gradient, q, sums of the p of each column)."""
    p = targets(indices, teacher, T)
    g, q, target = (np.zeros(logits.shape) for _ in range(3))
    for n in range(len(logits)):
        if not (indices[n] >= 0).any():
            continue
        e = np.exp((logits[n] - logits[n].max()) / T)
        q[n] = e / e.sum()
        for k, j in enumerate(indices[n]):
            if j >= 0:
                target[n, j] += p[n, k]
        g[n] = gl[n] * T * (q[n] - target[n])
    return g, q, target
