"""How near the distillation's sums come to the definition: errors that all terms of a row share do not average out."""
import numpy as np
import pytest
import torch

from test_gpu_decoder import dec, f64  # noqa: F401 (dec is a fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def rounding_of_factor(T):
    """How far log2(e) / T is moved by its rounding to fp32, relative."""
    k = 1.4426950408889634 / float(T)
    return float(np.float32(k)) / k - 1


def test_the_exponents_factor_has_no_bias(dec):
    """Two neighbouring temperatures whose factors log2(e) / T are rounded in opposite directions.  A factor that is off by r
    moves every exponential of a row the same way: the row's sum is off by r times the mean of (m - s) / T under its own
    weights, 8 here.  Errors of the additions differ from row to row: with their standard deviation below 3 U, the mean
    over 64 rows of the difference between the two temperatures is below 2.2 U (four deviations of 3 U sqrt(2 / 64)).
    Errors of the exponential itself are the same for both."""
    near = [np.float32(0.9 + 2.0 ** -24 * n) for n in range(20000)]
    low, high = min(near, key=rounding_of_factor), max(near, key=rounding_of_factor)
    assert rounding_of_factor(high) - rounding_of_factor(low) > 6e-8
    rng = np.random.default_rng(0)
    s = rng.uniform(-11.0, -7.0, (64, 100000)).astype(np.float32)
    s[:, 0] = 0.0
    index, teacher = torch.zeros(64, 1, dtype=torch.int64, device="cuda"), torch.zeros(64, 1, device="cuda")
    off = []
    for T in (low, high):
        stats = dec.distill_forward(torch.tensor(s).cuda(), index, teacher, float(T))[1]
        total = np.exp(s.astype(np.float64) / float(T)).sum(1)
        off.append((f64(stats)[:, 1] / total - 1).mean())
    assert abs(off[1] - off[0]) <= 2.2 * U, off


@pytest.mark.parametrize("T", [1.25, 2.0])
def test_row_sums_have_no_bias(dec, T):
    """The mean error of many rows' sums: the exponential's own, 5e-8 at the most on average (2^x of the hardware against 64
    bits, x in [-32, 0]: -0.2 to -0.9 U), once, whatever a thread and its neighbours find as their largest.  Errors that
    differ from row to row: a standard deviation below 3 U, of 256 rows four times 3 U / 16."""
    s = (torch.randn(256, 128000, generator=torch.Generator().manual_seed(0)) * 2.5).bfloat16().cuda()
    index, teacher = torch.zeros(256, 1, dtype=torch.int64, device="cuda"), torch.zeros(256, 1, device="cuda")
    stats = dec.distill_forward(s, index, teacher, T)[1]
    x = s.double()
    total = ((x - x.amax(1, keepdim=True)) / T).exp().sum(1)
    assert abs(float((stats[:, 1].double() / total - 1).mean())) <= (0.9 + 0.75) * U
