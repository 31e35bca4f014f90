"""Distillation at high temperatures, where the loss is a small difference of large terms."""
import numpy as np
import pytest
import torch

from test_gpu_decoder import DTYPES, IDS, check_distill, dec, f64, lists, randn  # noqa: F401 (dec is a fixture)

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -24, 2.0 ** -53
HIGH = [8.25, 20.0, 100.0, 1000.0, 2.0 ** 20]


def high_loss(s, i, t, T):
    """The loss from its definition with 64 bits of mantissa, whose own error is 2^-64 T^2 (log cols + 1) at the most (1e-5 of
    the smallest loss here), and a bound on the error of one computed in 53 bits from sums of exp(x) - 1, rounded to fp32.

    With a and b the differences to the largest over T, A and B the sums of their exponentials, loss / T^2 is sum p (a - b) +
    log(B / A).  A sum of n terms exp(b) - 1, each off by 6 E of itself, 50 times put under a larger maximum (4 E each),
    is off by (n + 206) E of the sum of min(1, |b|)."""
    x, y = s.astype(np.longdouble), t.astype(np.longdouble)
    loss, tol = np.zeros(len(x)), np.zeros(len(x))
    for n in range(len(x)):
        there = i[n] >= 0
        if not there.any():
            continue
        b = (x[n] - x[n].max()) / np.longdouble(T)
        a = (y[n][there] - y[n][there].max()) / np.longdouble(T)
        bl = b[i[n][there]]
        A, B = np.exp(a).sum(), np.exp(b).sum()
        p = np.exp(a) / A
        loss[n] = np.longdouble(T) ** 2 * ((p * (a - bl)).sum() + np.log(B / A))
        small = lambda v: np.minimum(1, np.abs(np.where(np.isfinite(v), v, 1))).sum()
        logs = (len(b) + 206) * small(b) / B + (len(a) + 206) * small(a) / A + 6 * (abs(len(b) - len(a)) + abs(float(B - A))) / B + 4 * abs(np.log(B / A))
        tol[n] = T * T * E * (logs + (len(a) + 20) * (p * (np.abs(a) + np.abs(bl))).sum()) + 1e-5 * abs(loss[n]) + 4 * U * abs(loss[n])
    return loss, tol


@pytest.mark.parametrize("T", HIGH)
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_loss_at_high_temperatures(dec, dtype, T):
    """Lists of all columns, of those that are not masked, and of some; rows of one part and of several."""
    for rows, cols, masked, top, ragged in [(6, 1000, 0, 1000, False), (5, 1017, 200, 817, False), (40, 300, 0, 16, True), (2, 70001, 1000, 1024, True), (700, 33, 0, 33, False)]:
        s = randn((rows, cols), dtype, cols, 2.5)
        s[:, cols - masked:] = float("-inf")
        if top == cols - masked:   # every column once, near to what the row has itself
            index = torch.stack([torch.randperm(top, generator=torch.Generator().manual_seed(r)) for r in range(rows)]).cuda()
            teacher = s.float().gather(1, index) + randn((rows, top), torch.float32, 7, 0.5)
        else:
            index, teacher = lists(rows, cols - masked, top, rows), randn((rows, top), torch.float32, 8, 2.0)
            if ragged:
                index[1] = -1
        loss, stats = dec.distill_forward(s, index, teacher, T)
        want, tol = high_loss(f64(s), index.cpu().numpy(), f64(teacher), T)
        off = np.abs(f64(loss) - want)
        assert (off <= tol).all(), (rows, cols, (off / np.maximum(np.abs(want), 1e-30)).max(), (off / np.maximum(tol, 1e-300)).max())
        if top == cols:   # a divergence
            assert bool((loss > 0).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS.get)
def test_sums_and_gradients_at_high_temperatures(dec, dtype):
    for T in HIGH[:4]:
        for rows, cols, top in [(7, 31, 5), (9, 1009, 8), (300, 257, 16), (2, 40000, 64)]:
            check_distill(dec, randn((rows, cols), dtype, cols, 2.5), lists(rows, cols, top, rows), randn((rows, top), torch.float32, top, 2.0), T)


def test_what_is_not_finite_at_a_high_temperature(dec):
    """As at any other: NaN (or +Inf) where the definition has no number, in that row alone."""
    s = randn((10, 400), torch.float32, 12, 2.0)
    index, teacher = lists(10, 400, 5, 13, ragged=False), randn((10, 5), torch.float32, 14)
    s[0, 17], s[1, 3], s[2, :] = float("nan"), float("inf"), float("-inf")
    s[3, :] = float("nan")
    index[3] = -1
    s[4, index[4, 0]] = float("-inf")
    s[5, index[5, 0]] = float("-inf")
    teacher[5, index[5] == index[5, 0]] = float("-inf")
    index[6, 2] = 400
    teacher[7, :] = float("-inf")
    s[8, :], teacher[8, :] = torch.finfo(torch.float32).min, 0.0   # uniform
    index[8] = torch.arange(5, device="cuda")
    loss, stats = dec.distill_forward(s, index, teacher, 20.0)
    assert loss.isnan().tolist() == [True, True, True, False, False, False, True, True, False, False]
    assert float(loss[3]) == 0.0 and float(loss[4]) == float("inf") and bool(loss[5].isfinite()) and float(stats[8, 1]) == 400.0
    assert abs(float(loss[8]) - 400.0 * np.log(400 / 5)) <= 4 * U * 400.0 * np.log(400 / 5)
