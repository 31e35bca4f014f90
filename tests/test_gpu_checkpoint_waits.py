"""Bounded waits of the checkpoint kernels where little work is left when one runs out.  In a build whose waits between
stages give up after one poll (-DAMPQ_TEST_SHORT_WAITS) a CTA ends with stages that were loaded and never multiplied: it waits
for their copies before it ends, so the kernels behind it find their shared memory untouched.  What was not stored is NaN,
everything else is right.  The build runs in processes of its own (AMPQ_LIBRARY picks it)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


def weight_gradients():
    """Six stages of work or fewer per tile (384 tokens in bf16, 128 in fp32), in pairs of CTAs and in single ones, one
    launch right behind the other."""
    import torch

    from paper_2505_13060_b200 import checkpoint as ckpt

    gave_up = 0
    for dtype, eps, sizes in ((torch.bfloat16, 2.0 ** -8, ((1, 300, 1536, 1792), (1, 384, 512, 520), (5, 257, 768, 1024), (2, 320, 4096, 4096))),
                              (torch.float32, 2.0 ** -24, ((1, 100, 1536, 2048), (1, 128, 2048, 2048), (3, 70, 1024, 1536)))):
        for samples, rows, cols, outs in sizes:
            g = torch.Generator(device="cuda").manual_seed(rows)
            x = torch.randn(samples * rows, cols, device="cuda", generator=g).to(dtype)
            gy = torch.randn(samples * rows, outs, device="cuda", generator=g).to(dtype)
            p = ckpt.pack(x)
            xd = ckpt.unpack(p, torch.float32).double().reshape(samples, rows, cols)
            gd = gy.double().reshape(samples, rows, outs)
            want, size = torch.matmul(gd.transpose(1, 2), xd), torch.matmul(gd.abs().transpose(1, 2), xd.abs())
            tol = (2 * rows + 8) * 2.0 ** -24 * size * 1.01 + eps * want.abs()
            for gw, gb in [ckpt.weight_grad(p, gy, samples=samples, bias=True) for _ in range(10)]:
                bad = torch.isnan(gw)
                assert bool((((gw.double() - want).abs() <= tol) | bad).all()), (dtype, samples, rows, cols, outs)
                assert bool(torch.isfinite(gb).all())
                gave_up += int(bad.any())
            q = ckpt.pack(x)
            assert torch.equal(p.codes, q.codes) and torch.equal(p.scales, q.scales)
    assert gave_up, "no wait ran out"
    print("gave up", gave_up)


def norms():
    """Rows that come by bulk copies, many to a group.  A row that a warp of its group missed has NaN outputs, and its
    checkpoint decodes to NaN or is right; the other rows are those of the same kernel fed by loads (rows off the 16-byte
    boundaries)."""
    import torch

    from paper_2505_13060_b200 import checkpoint as ckpt

    def odd(t):
        full = torch.empty(t.shape[0], t.shape[1] + 3, dtype=t.dtype, device="cuda")
        full[:, 1:-2] = t
        return full[:, 1:-2]

    gave_up = 0
    for dtype in (torch.bfloat16, torch.float32):
        for rows, cols in ((40000, 512), (20001, 1024), (9000, 4096), (5000, 5120), (3000, 8192), (2000, 16384)):
            g = torch.Generator(device="cuda").manual_seed(cols)
            x, gy = (torch.randn(rows, cols, device="cuda", generator=g).to(dtype) for _ in range(2))
            w = torch.rand(cols, device="cuda", generator=g).to(dtype)
            for kind in (0, 1):
                y, mean, rstd, p = ckpt.norm_forward(x, w, None, 1e-5, kind, 1)
                y2, mean2, rstd2, p2 = ckpt.norm_forward(odd(x), w, None, 1e-5, kind, 1)
                lost = torch.isnan(rstd)
                gave_up += int(lost.any())
                assert torch.equal(torch.isnan(y), lost[:, None].expand_as(y))
                codes, codes2 = p.codes.view(rows, -1, 32), p2.codes.view(rows, -1, 32)
                right = (p.scales == p2.scales) & (codes == codes2).all(2)
                assert bool((right | ((p.scales == 255) & (codes == 0).all(2) & lost[:, None])).all())
                kept = ~lost
                for a, b in ((y, y2), (rstd, rstd2)) + (((mean, mean2),) if kind == 0 else ()):
                    assert torch.equal(a[kept], b[kept]), (dtype, rows, cols, kind)
                if kind == 0:
                    assert torch.equal(torch.isnan(mean), lost)
                for base in (p2, x):
                    if base is x and dtype == torch.float32 and cols > 8192:
                        continue   # rows are read as they come
                    gx, gw, gb = ckpt.norm_backward(gy, base, mean2, rstd2, w, kind)
                    gx2, gw2, gb2 = ckpt.norm_backward(odd(gy), base, mean2, rstd2, w, kind)
                    lost = torch.isnan(gx).any(1)
                    gave_up += int(lost.any())
                    assert bool(torch.isnan(gx[lost]).all()) and torch.equal(gx[~lost], gx2[~lost])
                    for a, b in ((gw, gw2), (gb, gb2)) if kind == 0 else ((gw, gw2),):
                        assert bool((torch.isnan(a) | (a == b)).all())
    assert gave_up, "no wait ran out"
    print("gave up", gave_up)


@pytest.fixture(scope="module")
def short_waits(tmp_path_factory):
    from paper_2505_13060_b200 import build

    return build.build(out=str(tmp_path_factory.mktemp("short") / "libampq_short.so"), defines=["AMPQ_TEST_SHORT_WAITS"])


@pytest.mark.parametrize("what", ["weight_gradients", "norms"])
def test_waits_that_run_out(short_waits, what):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), what], env=dict(os.environ, AMPQ_LIBRARY=short_waits), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "gave up" in r.stdout


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    globals()[sys.argv[1]]()
