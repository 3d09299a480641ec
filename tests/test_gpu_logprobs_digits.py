"""Log probabilities of nearly certain rows and of very large logits, in every kind of block of the logits product.

Row n has the logit Z at one class (8 x, w in one column: a product of few bits, exact) and 0 at all others. So with C classes
rest = (C - 1) e^-Z, log p = -log1p(rest) of that class and d = -Z less that of the others, tau = -Z rest / (1 + rest), H = log1p(rest) - tau.
Tolerances, relative: an exponential is off by |d| 2^-22 for the product with log2 e and the exponent's own rounding, 2^-21 for the base-2 unit,
and its sums by (tiles / 256 + 64) 8 u, u = 2^-24: e in all. H, log p and tau are sums and quotients of such terms, of one sign:
2 e + 4 u. The gradient in a logit has a term of g and one of h, each off by that (8 u for its few operations); bf16 models round it
once (2^-8) and the gradient in x, which has one product here, once more; where the exponentials are kept, 2^-11 of p and of d as f16 has
them, and 2^-40 for what f16 cannot hold.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from test_gpu_logprobs import forward, grad
from test_gpu_softmax_loss import DT, U, handle, held

pytestmark = pytest.mark.gpu

# whole tiles: streamed blocks, 64 x 64, 128 x 128 in two forms, 256 x 256, and the blocks of few rows
SIZES = [(16, 64, 4096), (300, 64, 4096), (4096, 64, 8192), (1024, 1024, 2688), (1024, 1024, 8192), (50, 64, 100096),
         (64, 64, 40064), (9, 64, 30784)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", SIZES)
def test_nearly_certain_rows_keep_their_digits(dtype, rows, dim, classes):
    need_gpu()
    print("logprobs nearly certain", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    g = torch.Generator().manual_seed(4)
    n, k = torch.arange(rows), min(64, rows, dim)
    s, y = 0.75, torch.randperm(classes, generator=g)[:k]
    b = torch.linspace(0.5, 50.0 / 6, k).to(DT[dtype])
    x, w = torch.zeros(rows, dim), torch.zeros(classes, dim)
    x[n, n % k] = 8.0
    w[y, torch.arange(k)] = b.float()
    mine = n % 3 < 2                                       # whose label is the likely class; the others' is the next one's
    labels = torch.where(mine, y[n % k], y[(n + 1) % k])
    up, uh = torch.where(mine, torch.randn(rows, generator=g), 0.0) / rows, torch.randn(rows, generator=g) / rows
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=labels.cuda(), off=None, s=s, g=up.cuda(), h=uh.cuda())
    up, uh = up.double(), uh.double()
    Z = s * 8.0 * b.double()[n % k]
    p = torch.exp(-Z)
    rest = (classes - 1) * p
    log_all, tau = torch.log1p(rest), -Z * rest / (1 + rest)
    H = log_all - tau
    e = Z * 2.0 ** -22 + 2.0 ** -21 + (classes / 16 / 256 + 64) * 8 * U
    rel = (2 * e + 4 * U) * (1 + 2.0 ** -4)
    # the gradient in the logits at the k classes that stand in a column of w, and its terms' sizes
    G = p[:, None] * (-up[:, None] - uh[:, None] * (-Z - tau)[:, None]).expand(rows, k) / (1 + rest)[:, None]
    size = p[:, None] * (up.abs()[:, None] + uh.abs()[:, None] * (Z + tau.abs())[:, None]).expand(rows, k) / (1 + rest)[:, None]
    G, size = G.clone(), size.clone()
    G[n, n % k] = (up * rest + uh * tau) / (1 + rest)
    size[n, n % k] = (up.abs() * rest + uh.abs() * tau.abs()) / (1 + rest)
    want = s * G * b.double()
    for keep in (False, True):
        out = forward(lib, c, rows, dim, classes, 1, keep)
        held("entropy", out["entropy"].cpu(), H, rel * H)
        held("logprob", out["logprob"].cpu()[mine], -log_all[mine], rel[mine] * log_all[mine])
        assert torch.equal(out["top_ids"].cpu()[:, 0], y[n % k])
        held("top_logprob", out["top_logprob"].cpu()[:, 0], -log_all, rel * log_all)
        gx, _ = grad(lib, c, rows, dim, classes, out)
        bound = size * (rel + 8 * U)[:, None]
        if keep and dtype == "bf16":
            bound = bound + size * 2.0 ** -11 + (up.abs() + uh.abs() * (Z + 2))[:, None] * 2.0 ** -40 + \
                (uh.abs() * p / (1 + rest))[:, None] * 2.0 ** -10
            bound[n, n % k] = (size * (rel + 8 * U)[:, None])[n, n % k]  # (its exponential is 1)
        bound = s * bound * b.double()
        r = 2.0 ** -8 if dtype == "bf16" else U
        bound = bound * (1 + r) ** 2 + want.abs() * (2 * r + r * r) + 1e-37
        held("grad_x", gx.cpu()[:, :k], want, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", SIZES + [(300, 64, 4090), (1000, 64, 20000)])
def test_very_large_logits(dtype, rows, dim, classes):
    """Rows of one large negative logit for every class (log p = -log C, H = log C), rows with one class far above the others (log p = 0 or
    minus all of the logit, H = 0), and ordinary ones beside them, which are the same to the bit without the others. The large logits are products of two
    powers of two, the uniform rows' p = 1 / C, off by 2^-20 for the sums (64 chains of at most 8 u of a tile's terms) and 2 u of itself; gradients add 2
    halves of a step, and their sums of C products that cancel nothing (C / 4 + 40) u."""
    need_gpu()
    print("logprobs very large", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    g = torch.Generator().manual_seed(5)
    s, big = 0.75, 2.0 ** 17
    x, w = torch.randn(rows, dim, generator=g), torch.randn(classes, dim, generator=g) * 0.2
    n, one = torch.arange(rows), classes // 3
    kind = n % 3
    x[:, :2] = 0.0
    w[:, 0], w[:, 1] = -big, 0.0
    w[one, 1] = big
    x[kind < 2] = 0.0
    x[kind == 0, 0] = big
    x[kind == 1, 1] = big
    y = torch.randint(0, classes, (rows,), generator=g)
    y[kind == 1] = torch.where(n[kind == 1] % 2 == 0, one, one + 1)
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=y.cuda(), off=None, s=s,
             g=(torch.randn(rows, generator=g) / rows).cuda(), h=(torch.randn(rows, generator=g) / rows).cuda())
    plain = dict(c, x=c["x"].clone())
    plain["x"][(kind < 2).cuda()] = 0.0
    z, log_c = s * big * big, math.log(classes)
    tol = 2.0 ** -20 + (classes / 16 / 256 + 64) * 8 * U
    for keep in (False, True):
        out, ref = forward(lib, c, rows, dim, classes, 2, keep), forward(lib, plain, rows, dim, classes, 2, keep)
        gx, gw = grad(lib, c, rows, dim, classes, out)
        gp, _ = grad(lib, plain, rows, dim, classes, ref)
        get = lambda k, q: out[k].cpu()[kind == q].double()
        for k in ("logprob", "entropy", "lse", "top_ids", "top_logprob"):
            assert torch.equal(out[k].cpu()[kind == 2], ref[k].cpu()[kind == 2]), k
        assert torch.equal(gx.cpu()[kind == 2], gp.cpu()[kind == 2])
        full = lambda v: torch.full((int((kind == 0).sum()),), v, dtype=torch.float64)
        for k, v in (("logprob", -log_c), ("entropy", log_c), ("lse", log_c - s * big * big)):
            held(k, get(k, 0), full(v), full(tol * log_c + 2 * U * abs(v)))
        assert torch.equal(out["top_ids"].cpu()[kind == 0], torch.tensor([0, 1]).expand(int((kind == 0).sum()), 2))
        assert (get("entropy", 1) == 0).all()
        assert torch.equal(get("logprob", 1), torch.where(y[kind == 1] == one, 0.0, -z).double())
        assert (out["top_ids"].cpu()[kind == 1, 0] == one).all() and (get("top_logprob", 1)[:, 0] == 0).all()
        assert torch.isfinite(gx.float()).all() and torch.isfinite(gw.float()).all()
        # s g (w[y] - the mean of w) for uniform rows, whose entropy is the largest there is
        up, mean = c["g"].cpu().double()[kind == 0, None], c["w"].cpu().double().mean(0)
        wa = c["w"].cpu().double().abs().mean(0)
        wy = c["w"].cpu().double()[y[kind == 0]]
        uh = c["h"].cpu().double()[kind == 0, None]
        want = s * up * (wy - mean)
        r = 2.0 ** -8 if dtype == "bf16" else U
        half = 2.0 ** -10 if keep and dtype == "bf16" else 0.0  # (p and d as f16 has them)
        e = tol + 8 * U + half + (classes / 4 + 40) * 2 * U
        bound = s * ((up.abs() * (wa + wy.abs())) * (e + r) + uh.abs() * wa * (e * (1 + log_c))) * (1 + r) + r * want.abs() + 1e-37
        held("grad_x", gx.cpu()[kind == 0], want, bound * (1 + 2.0 ** -4))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", SIZES + [(300, 64, 4090), (1000, 64, 20000)])
@pytest.mark.parametrize("low", [-math.inf, -3e38])
def test_one_logit_far_below_all_others(dtype, rows, dim, classes, low):
    """A logit of -inf, or one whose product with log2 e is, counts as that of a masked class."""
    need_gpu()
    print("logprobs one far below", dtype, rows, dim, classes, low, flush=True)
    lib = handle(dtype)
    g = torch.Generator().manual_seed(9)
    at = classes // 2
    x, w = torch.randn(rows, dim, generator=g), torch.randn(classes, dim, generator=g) * 0.2
    x[:, 0] = 1.0
    y = torch.randint(0, at, (rows,), generator=g)
    c = dict(x=x.to(DT[dtype]).cuda(), w=w.to(DT[dtype]).cuda(), y=y.cuda(), off=None, s=1.0)
    c["w"][at, 0] = low
    for keep in (False, True):
        out = forward(lib, c, rows, dim, classes, 4, keep)
        z = c["x"].double() @ c["w"].double().t().contiguous()
        lp = torch.log_softmax(z, 1)
        H = -(lp.exp() * lp.masked_fill(torch.isneginf(lp), 0.0)).sum(1)
        # dz as derived beside the operator's other tests: (dim / 4 + 20 [+ dim]) u of the sums of sizes; e of every exponential, as above
        keepers = torch.arange(classes, device="cuda") != at
        size = (c["x"].double().abs() @ c["w"].double().abs()[keepers].t().contiguous()).amax(1)
        dz = (dim / 4 + 20 + (dim if dtype == "f32" else 0)) * U * size
        span = (z[:, keepers].amax(1) - z[:, keepers].amin(1))
        e = 2 * dz + span * 2.0 ** -22 + 2.0 ** -21 + (classes / 16 / 256 + 64) * 8 * U
        held("entropy", out["entropy"], H, (2 * e * (1 + H + span) + 4 * U * H) * (1 + 2.0 ** -4))
        want = lp.gather(1, c["y"][:, None])[:, 0]
        held("logprob", out["logprob"], want, (e + 2 * dz + 4 * U * want.abs()) * (1 + 2.0 ** -4))
        assert (out["top_ids"] != at).all() and (out["top_ids"] >= 0).all()
