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
         (64, 64, 40064), (9, 64, 30720)]


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
