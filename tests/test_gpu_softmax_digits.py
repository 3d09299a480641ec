"""Softmax loss where a row's float log-sum-exp has too few digits: labels of probability close to 1, whose loss and gradient
are about 1 - p, and logits that all lie far from 0 (an offset that every class has). Inputs are made so that each logit
is a single product, and the label's gradient can be read off alone.

Tolerances (u = 2^-24). A logit s a b is off by 2 u |z| (one product of two factors that are exact, times s). With R the sum
of the other classes' exponentials and e the label's, 1 - p = R / (R + e) and loss = log(1 + R / e): a difference of logits enters the exponent, so
4 u |z| of themselves; exponentials of arguments x down to -40 are off by |x| u + 2^-21 at most, three of them in a row (tile, join,
label), and the sums and quotients by 2^-19 for the sizes here: 4 u |z| + 3 (40 u + 2^-21) + 2^-19 < 4 u |z| + 2^-16. bf16 models round
the label's element of G to bf16 once (2^-8); what multiplies it is a power of two and the other terms are zeros, so the gradient is that value.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn
from test_gpu_softmax_loss import DT, U, call_forward, call_grad_within, handle, held

pytestmark = pytest.mark.gpu


def sharp(dtype, rows, classes, seed=0):
    """Row n's logits are 0 but for its label's, which makes 1 - p run from 10^-1 to 10^-9 over the rows. In column rows + n of w
    only the label's class of row n has a value (1)."""
    g = torch.Generator().manual_seed(seed)
    dim, a, s = 2 * rows + 8, 8.0, 0.75
    y = torch.randperm(classes, generator=g)[:rows]
    rest = 10.0 ** -torch.linspace(1, 9, rows, dtype=torch.float64)
    b = (torch.log((classes - 1) / rest) / (a * s)).to(DT[dtype])
    x, w = torch.zeros(rows, dim), torch.zeros(classes, dim)
    n = torch.arange(rows)
    x[n, n] = a
    w[y, n] = b.float()
    w[y, rows + n] = 1.0
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=y.cuda(), off=None, wt=None, s=s, scale=0.5)
    return c, dim, s * a * b.double()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,classes", [(16, 4096), (120, 3001), (300, 9000), (1024, 8192)])
def test_labels_near_probability_one(dtype, rows, classes):
    need_gpu()
    print("softmax digits", dtype, rows, classes, flush=True)
    lib = handle(dtype)
    c, dim, z = sharp(dtype, rows, classes)
    ratio = (classes - 1) * torch.exp(-z)  # R / e
    want, miss = torch.log1p(ratio), ratio / (1 + ratio)
    assert float(miss.min()) < 2e-9 and float(miss.max()) > 0.05
    tol = 4 * U * z + 2.0 ** -16
    f = c["s"] * c["scale"]
    n = torch.arange(rows)
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    assert least < most
    loss, _ = call_forward(lib, c, rows, dim, classes)
    losses = [loss]
    for size in (most, least):
        loss, _, gx, gw = call_grad_within(lib, c, rows, dim, classes, size)
        losses.append(loss)
        r = tol + (2.0 ** -8 * (1 + 2.0 ** -15) if dtype == "bf16" else U)
        held("grad_x at the label, %d bytes" % size, gx.cpu()[n, rows + n], -f * miss, r * f * miss)
        # (x's value, 8, is a power of two)
        held("grad_w at the label, %d bytes" % size, gw.cpu()[c["y"].cpu(), n], -8 * f * miss, r * 8 * f * miss)
    for loss in losses:
        held("loss", loss.cpu(), want, tol * want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [-1e9, 3e7, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("rows", [40, 300])
def test_an_offset_that_every_class_has(dtype, value, rows):
    """All logits are that number, so every class has probability 1 / V: x has zeros where w has values and the other way round."""
    need_gpu()
    print("softmax common offset", dtype, value, rows, flush=True)
    lib = handle(dtype)
    dim, classes = 64, 5003
    g = torch.Generator().manual_seed(3)
    x, w = torch.zeros(rows, dim), torch.zeros(classes, dim)
    x[:, :32] = torch.randn(rows, 32, generator=g)
    w[:, 32:] = torch.randn(classes, 32, generator=g)
    y = torch.randint(0, classes, (rows,), generator=g).cuda()
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=y, off=torch.full((classes,), value, device="cuda"),
             wt=None, s=1.0, scale=0.25)
    G = torch.full((rows, classes), 0.25 / classes, dtype=torch.float64, device="cuda")
    G[torch.arange(rows), y] -= 0.25
    xd, wd = c["x"].double(), c["w"].double()
    ref_x, ref_w = G @ wd, G.t().contiguous() @ xd
    # half a step of f16 and of bf16 for each element of G, the sums (float), a half step of the result
    r, half = (2.0 ** -8 + 2.0 ** -10, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -19, U)
    chain = (classes / 4 + 40) * 2 * U
    bx = (G.abs() @ wd.abs()) * (r + chain)
    bw = (G.abs().t().contiguous() @ xd.abs()) * (r + chain)
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    assert least < most
    want = torch.full((rows,), math.log(classes), dtype=torch.float64, device="cuda")
    for size in (most, least):
        loss, lse, gx, gw = call_grad_within(lib, c, rows, dim, classes, size)
        held("loss", loss, want, 2.0 ** -19 * want)
        held("lse", lse, want + value, 2 * U * abs(value) + 2.0 ** -19 * want)
        held("grad_x", gx, ref_x, bx + half * (ref_x.abs() + bx))
        held("grad_w", gw, ref_w, bw + half * (ref_w.abs() + bw))
    loss, _ = call_forward(lib, c, rows, dim, classes)
    held("loss", loss, want, 2.0 ** -19 * want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_lowest_value_masks_like_minus_infinity(dtype):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 200, 64, 5003
    g = torch.Generator().manual_seed(4)
    off = torch.randn(classes, generator=g)
    masked = torch.rand(classes, generator=g) < 0.5
    masked[1024:2048] = True  # whole tiles, and a whole piece
    y = torch.nonzero(~masked)[:, 0][torch.randint(0, int((~masked).sum()), (rows,), generator=g)].cuda()
    c = dict(x=torch.randn(rows, dim, generator=g).to(DT[dtype]).cuda(), y=y, wt=None, s=0.75, scale=0.25,
             w=(torch.randn(classes, dim, generator=g) * 0.3).to(DT[dtype]).cuda())
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    for size in (most, least):
        got = []
        for value in (-math.inf, torch.finfo(torch.float32).min):
            o = off.clone()
            o[masked] = value
            got.append(call_grad_within(lib, dict(c, off=o.cuda()), rows, dim, classes, size))
        assert all(torch.equal(a, b) for a, b in zip(*got))
        assert (got[1][3][masked.cuda()] == 0).all() and torch.isfinite(got[1][0]).all()
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,classes", [(12, 50), (40, 1500), (200, 1301), (700, 1025)])
def test_the_other_classes_of_labels_near_probability_one(dtype, rows, classes):
    """Every class's gradient in the logits, read off in a column of its own (w has 1 there), where the label is up to e^-50 of the
    way to 1: the classes beside it in a tile keep their digits too. f p for each of the others, with the tolerance above and, for
    bf16, half a step of f16 (2^-11) besides that of bf16."""
    need_gpu()
    print("softmax digits of all classes", dtype, rows, classes, flush=True)
    lib = handle(dtype)
    g = torch.Generator().manual_seed(1)
    n = torch.arange(rows)
    dim = (classes + rows + 7) // 8 * 8
    y = torch.randint(0, classes, (rows,), generator=g)
    b = torch.linspace(0.5, 50.0 / 6, rows).to(DT[dtype])
    x, w = torch.zeros(rows, dim), torch.zeros(classes, dim)
    x[n, classes + n] = 8.0
    w[torch.arange(classes), torch.arange(classes)] = 1.0
    w[y, classes + n] = b.float()
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=y.cuda(), off=None, wt=None, s=0.75, scale=0.5)
    z = torch.zeros(rows, classes, dtype=torch.float64)
    z[n, y] = 0.75 * 8.0 * b.double()
    p = torch.softmax(z, 1)
    miss = (classes - 1) * torch.exp(-z[n, y])
    p[n, y] = -miss / (1 + miss)
    want = 0.75 * 0.5 * p
    tol = 4 * U * z.amax(1, keepdim=True) + 2.0 ** -16 + ((1 + 2.0 ** -8) * (1 + 2.0 ** -11) - 1 if dtype == "bf16" else 2 * U)
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    for size in (most, least):
        _, _, gx, _ = call_grad_within(lib, c, rows, dim, classes, size)
        held("grad_x, %d bytes" % size, gx.cpu()[:, :classes], want, tol * want.abs())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,classes", [(40, 33), (40, 5003), (300, 2001), (1000, 20000)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_row_that_is_not_finite_is_not_hidden(dtype, rows, classes, value):
    """Its loss, lse and gradient are NaN, and with them grad_w, so that the norm of the gradients sees it; other rows' results are
    those of a batch without it."""
    need_gpu()
    lib = handle(dtype)
    dim = 64
    g = torch.Generator().manual_seed(6)
    c = dict(x=torch.randn(rows, dim, generator=g).to(DT[dtype]).cuda(), off=None, wt=None, s=0.75, scale=0.25,
             w=(torch.randn(classes, dim, generator=g) * 0.3).to(DT[dtype]).cuda(),
             y=torch.randint(0, classes, (rows,), generator=g).cuda())
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    for size in sorted({most, least}):
        clean = call_grad_within(lib, c, rows, dim, classes, size)
        x = c["x"].clone()
        x[7] = value
        got = call_grad_within(lib, dict(c, x=x), rows, dim, classes, size)
        for a, b in zip(got[:3], clean[:3]):
            assert torch.isnan(a[7]).all() and torch.isfinite(b).all()
            a[7] = b[7]
            assert torch.equal(a, b)
        assert torch.isnan(got[3]).any()
        loss, lse = call_forward(lib, dict(c, x=x), rows, dim, classes)
        assert torch.isnan(loss[7]) and torch.isnan(lse[7]) and int(torch.isnan(loss).sum()) == 1
