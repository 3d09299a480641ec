"""Log probabilities and Muon where places pass 2^31 elements, and 2^24 rows: samples of the results against their definition in 64 bits.

Log probabilities: with dim 64 a logit is off by dz = (dim / 4 + 20) u of the sums of sizes (u = 2^-24), an exponential by 2 dz + |d| 2^-22 + 2^-21 and
its sums by (tiles / 256 + 64) 8 u; gradients are summed from elements rounded to bf16 (2^-8) and, kept, to f16 (2^-11 of p and of d), rounded once more.
Muon: five steps' 2e-4 of X's norm, as derived in test_gpu_muon_spectra.py, of a sample of its rows with 6 times that, as errors are spread evenly.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from test_gpu_logprobs import forward, grad, upstream
from test_gpu_muon import ABC, handle as muon_handle, step
from test_gpu_softmax_loss import U, handle, held, make

pytestmark = pytest.mark.gpu


def room(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30:
        pytest.skip("needs %d GiB of device memory" % gigabytes)


@pytest.mark.parametrize("keep", [True, False])
def test_more_than_2_to_32_logits(keep):
    need_gpu()
    room(60)
    rows, dim, classes, top = 33000, 64, 131072 + 8, 3
    assert rows * classes > 2 ** 32
    lib = handle("bf16")
    c = upstream(make("bf16", rows, dim, classes, 3), rows, 4)
    out = forward(lib, c, rows, dim, classes, top, keep)
    gx, gw = grad(lib, c, rows, dim, classes, out)
    torch.cuda.synchronize()
    w, last = c["w"].double(), 40
    wa = w.abs()
    want_w, sizes = torch.zeros(last, dim, dtype=torch.float64, device="cuda"), torch.zeros(last, dim, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 1000):
        here = slice(at, at + 1000)
        x, y = c["x"][here].double(), c["y"][here]
        z = c["s"] * (x @ w.t().contiguous())
        m = z.amax(1, keepdim=True)
        lse = torch.exp(z - m).sum(1, keepdim=True).log() + m
        lp = z - lse
        p = lp.exp()
        H = -(p * lp).sum(1, keepdim=True)
        g, h = c["g"][here].double()[:, None], c["h"][here].double()[:, None]
        size = c["s"] * (x.abs() @ wa.t().contiguous()).amax(1)
        dz = (dim / 4 + 20) * U * size
        span = (m - z.amin(1, keepdim=True))[:, 0]
        e = 2 * dz + span * 2.0 ** -22 + 2.0 ** -21 + (classes / 16 / 256 + 64) * 8 * U
        held("lse", out["lse"][here], lse[:, 0], dz + e + 2 * U * lse[:, 0].abs())
        want = lp.gather(1, y[:, None])[:, 0]
        held("logprob", out["logprob"][here], want, e + 2 * dz + 4 * U * want.abs())
        held("entropy", out["entropy"][here], H[:, 0], 2 * e * (1 + H[:, 0] + span))
        best = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top] if at + 1000 >= rows else None
        if best is not None:
            assert torch.equal(out["top_ids"][here], best)
        live = (g != 0) | (h != 0)
        hot = torch.zeros_like(z).scatter_(1, y[:, None], 1.0)
        G = torch.where(live, c["s"] * (g * (hot - p) - h * p * (lp + H)), 0.0)
        Ga = c["s"] * (g.abs() * (hot * (1 - p) + p * (1 - hot)) + h.abs() * p * ((lp + H).abs() + 2 * H))
        r = 2.0 ** -8
        f = r + 2 * e.max().item() + (classes / 4 + 40) * U + (2.0 ** -9 if keep else 0.0)
        flat = (g.abs() + h.abs() * 30) * p.amax(1, keepdim=True) * 2.0 ** -40 * c["s"]
        want_w += G[:, -last:].t().contiguous() @ x
        sizes += (Ga[:, -last:] * f + flat).t().contiguous() @ x.abs()
        if at == 0 or at + 1000 >= rows:
            wx = G @ w
            held("grad_x", gx[here], wx, ((Ga * f + flat) @ wa) * (1 + r) + r * wx.abs() + 1e-30)
    held("grad_w", gw[-last:], want_w, sizes * (1 + r) + r * want_w.abs() + 1e-30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_2_to_24_rows(dtype):
    need_gpu()
    room(40)
    rows, dim, classes, top = 1 << 24, 8, 9, 2
    lib = handle(dtype)
    c = upstream(make(dtype, rows, dim, classes, 5), rows, 6)
    out = forward(lib, c, rows, dim, classes, top, True)
    gx, _ = grad(lib, c, rows, dim, classes, out)
    torch.cuda.synchronize()
    for at in (0, rows // 2 + 1, rows - 1000):
        here = slice(at, at + 1000)
        x, w, y = c["x"][here].double(), c["w"].double(), c["y"][here]
        z = c["s"] * (x @ w.t().contiguous())
        lp = torch.log_softmax(z, 1)
        H = -(lp.exp() * lp).sum(1, keepdim=True)
        want = lp.gather(1, y[:, None])[:, 0]
        span = z.amax(1) - z.amin(1)
        dz = (dim / 4 + 20 + dim) * U * c["s"] * (x.abs() @ w.abs().t().contiguous()).amax(1)
        e = 2 * dz + span * 2.0 ** -22 + 2.0 ** -21 + 66 * 8 * U
        held("logprob", out["logprob"][here], want, e + 2 * dz + 4 * U * want.abs())
        held("entropy", out["entropy"][here], H[:, 0], 2 * e * (1 + H[:, 0] + span))
        assert torch.equal(out["top_ids"][here], torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top])
        g, h = c["g"][here].double()[:, None], c["h"][here].double()[:, None]
        hot, p = torch.zeros_like(z).scatter_(1, y[:, None], 1.0), lp.exp()
        G = c["s"] * (g * (hot - p) - h * p * (lp + H))
        Ga = c["s"] * (g.abs() * (hot * (1 - p) + p * (1 - hot)) + h.abs() * p * ((lp + H).abs() + 2 * H))
        r = 2.0 ** -8 if dtype == "bf16" else U
        bound = (Ga @ w.abs()) * (r + 2 * e.max().item() + 50 * U + (2.0 ** -9 if dtype == "bf16" else 0.0)) * (1 + r) + r * (G @ w).abs() + 1e-30
        held("grad_x", gx[here], G @ w, bound)


@pytest.mark.parametrize("rows,cols", [(1 << 20, 2100), (2100, (1 << 20) - 3)])
def test_matrices_of_more_than_2_to_31_elements(rows, cols):
    need_gpu()
    room(130)
    assert rows * cols > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(2)
    lib = muon_handle()
    t = dict(param=torch.zeros(rows, cols, device="cuda"), m=torch.zeros(rows, cols, device="cuda"), weight_decay=0.0, scale=-1.0,
             grad=torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.float32).bfloat16())
    step(lib, [t], momentum=0.0, nesterov=False)
    torch.cuda.synchronize()
    u, x = t["grad"], t["param"]
    assert torch.equal(t["m"][-3:], u[-3:].float())
    tall = rows > cols
    short = min(rows, cols)
    # the Gram matrix in 64 bits, and the polynomial P of it: X = P U / |U|, or U P / |U|
    gram, norm = torch.zeros(short, short, dtype=torch.float64, device="cuda"), 0.0
    for at in range(0, max(rows, cols), 1 << 16):
        part = (u[at:at + (1 << 16)] if tall else u[:, at:at + (1 << 16)].t()).double().contiguous()
        gram += part.t().contiguous() @ part
        norm += float((part * part).sum())
    a, b, c = ABC
    A, P, eye = gram / norm, torch.eye(short, dtype=torch.float64, device="cuda"), torch.eye(short, dtype=torch.float64, device="cuda")
    for _ in range(5):
        T = a * eye + b * A + c * (A @ A)
        P, A = T @ P, T @ A @ T
    for where in (slice(0, 500), slice(max(rows, cols) - 501, max(rows, cols))):
        part = (u[where] if tall else u[:, where].t()).double().contiguous() / math.sqrt(norm)
        want = part @ P
        got = (x[where] if tall else x[:, where].t()).double()
        assert float((got - want).norm()) <= 6 * 2e-4 * float(want.norm())
