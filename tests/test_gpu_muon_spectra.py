"""The Muon step's accuracy over spectra from even to steep, in both kinds of kernels (one workgroup a matrix, and launches of blocks).

Tolerance of X after k steps of the default coefficients, relative in the 2-norm: a pair of f16 is off by up to 2^-23 of a value, e = 2^-23 /
sqrt(3) = 6.9e-8 where roundings are as good as random. A step's errors, relative to |X|: those of A times |b| (what its large directions leak into
others), of T times a, and of X: (4.8 + 3.4 + 1) e = 6.4e-7; the float sums of the products lie below (2^-24 of partial sums). Whatever has entered
grows by at most a = 3.4445, the slope at 0, in each later step, so that 6.4e-7 (1 + a + .. + a^(k-1)) + e a^k is left of |X0| = 1, against an X
of one singular value at least 0.7: for five steps 2.3e-4 with all added up, 2e-4 in quadrature with X0's own part. So TOL(k) = 2e-4 a^(k - 5).
"""
import pytest
import torch

from gpu_helpers import need_gpu
from test_gpu_muon import ABC, handle, newton_schulz, step

pytestmark = pytest.mark.gpu


def spectrum(kind, m):
    i = torch.arange(m, dtype=torch.float64)
    if kind == "even":
        return torch.ones(m, dtype=torch.float64)
    if kind == "one large":
        return torch.where(i == 0, 1.0, 1e-4).double()
    if kind == "half large":
        return torch.where(i < m // 2, 1.0, 1e-3).double()
    return (i + 1) ** -float(kind[3:]) if kind.startswith("i^-") else 10.0 ** (-float(kind[4:]) * i / (m - 1))


@pytest.mark.parametrize("rows,cols", [(30, 80), (64, 64), (96, 200), (200, 96), (500, 700), (1000, 1000)])
@pytest.mark.parametrize("kind", ["even", "one large", "half large", "i^-0.5", "i^-2", "10^-3", "10^-6"])
def test_update_over_spectra(rows, cols, kind):
    need_gpu()
    lib = handle()
    g = torch.Generator().manual_seed(rows)
    m = min(rows, cols)
    u, _ = torch.linalg.qr(torch.randn(rows, m, generator=g, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(cols, m, generator=g, dtype=torch.float64))
    grad = ((u * spectrum(kind, m)) @ v.t()).float()
    for steps in (1, 2, 3, 5, 6, 8):
        t = dict(param=torch.zeros(rows, cols, device="cuda"), grad=grad.cuda(), m=torch.zeros(rows, cols, device="cuda"),
                 weight_decay=0.0, scale=-1.0)
        step(lib, [t], momentum=0.0, nesterov=False, steps=steps)
        ref = newton_schulz(grad, steps=steps)
        off = float((t["param"].double() - ref).norm() / ref.norm())
        assert off <= 2e-4 * ABC[0] ** (steps - 5), "%d steps: %.3g" % (steps, off)


@pytest.mark.parametrize("abc", [(2.0, -1.5, 0.5), (1.875, -1.25, 0.375), (3.0, -3.0, 1.0), (-3.4445, 4.7750, -2.0315)])
@pytest.mark.parametrize("rows,cols", [(48, 80), (130, 300)])
@pytest.mark.parametrize("kind", ["even", "one large", "i^-0.5", "10^-3"])
def test_other_coefficients(abc, rows, cols, kind):
    """The same sum with these coefficients' |a| and |b|, all added up."""
    need_gpu()
    lib = handle()
    g = torch.Generator().manual_seed(1)
    m = min(rows, cols)
    u, _ = torch.linalg.qr(torch.randn(rows, m, generator=g, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(cols, m, generator=g, dtype=torch.float64))
    grad = ((u * spectrum(kind, m)) @ v.t()).float()
    e, a = 2.0 ** -23 / 3 ** 0.5, abs(abc[0])
    for steps in (1, 2, 3, 4, 5, 8, 12):
        t = dict(param=torch.zeros(rows, cols, device="cuda"), grad=grad.cuda(), m=torch.zeros(rows, cols, device="cuda"),
                 weight_decay=0.0, scale=-1.0)
        step(lib, [t], momentum=0.0, nesterov=False, steps=steps, coefficients=abc)
        ref = newton_schulz(grad, abc, steps)
        off = float((t["param"].double() - ref).norm() / ref.norm())
        assert off <= ((a + abs(abc[1]) + 1) * e * sum(a ** i for i in range(steps)) + e * a ** steps) / 0.7, "%d steps: %.3g" % (steps, off)
