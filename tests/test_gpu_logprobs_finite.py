"""Log probabilities of rows whose logits are not finite: NaN or +inf is not hidden by a maximum or by a clamp, wherever it stands."""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn
from test_gpu_logprobs import forward, grad, upstream
from test_gpu_softmax_loss import handle, make

pytestmark = pytest.mark.gpu

# every kind of block of the logits product, whole ones and ragged ones (rows, dim, classes)
SIZES = [(9, 16, 1), (40, 64, 33), (40, 64, 5003), (300, 64, 2048), (300, 64, 2001), (1000, 64, 20000), (1024, 1024, 2688),
         (1024, 512, 20000), (50, 64, 100096), (40, 72, 40001), (9, 64, 30784)]


def results(lib, c, rows, dim, classes, top):
    for keep in (False, True):
        out = forward(lib, c, rows, dim, classes, top, keep)
        gx, gw = grad(lib, c, rows, dim, classes, out)
        torch.cuda.synchronize()
        yield out, gx, gw


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", SIZES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_a_row_that_is_not_finite_is_not_hidden(dtype, rows, dim, classes, value, masked):
    """Its results are NaN, its gradient too, and with them grad_w; other rows' results are those of a batch without it."""
    need_gpu()
    print("logprobs not finite", dtype, rows, dim, classes, value, masked, flush=True)
    lib = handle(dtype)
    top = min(4, classes)
    c = upstream(make(dtype, rows, dim, classes, 6, masked=masked), rows, 3)
    if masked:
        c["off"][classes // 2:classes // 2 + 70] = -math.inf  # a tile without any class
        c["off"][0] = 0.25
        c["y"][:] = 0
    bad = dict(c, x=c["x"].clone())
    bad["x"][7] = value
    for labels in (True, False):
        if not labels:
            c, bad = dict(c, y=None, g=None), dict(bad, y=None, g=None)
        for (a, ax, aw), (b, bx, bw) in zip(results(lib, bad, rows, dim, classes, top), results(lib, c, rows, dim, classes, top)):
            for k in ("logprob", "entropy", "lse"):
                if a[k] is not None:
                    assert torch.isnan(a[k][7]) and not torch.isnan(b[k]).any(), k
                    a[k][7] = b[k][7]
                    assert torch.equal(a[k], b[k]), k
            ids = a["top_ids"][7]
            assert ((ids >= -1) & (ids < classes)).all()
            for k in ("top_ids", "top_logprob"):
                a[k][7] = b[k][7]
                assert torch.equal(a[k], b[k]), k
            assert torch.isnan(ax[7]).all() and torch.isfinite(bx.float()).all()
            ax[7] = bx[7]
            assert torch.equal(ax, bx)
            assert torch.isnan(aw).any() and torch.isfinite(bw.float()).all()
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", [s for s in SIZES if s[2] > 1])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_one_logit_that_is_not_finite(dtype, rows, dim, classes, value):
    """One class's weights hold it: every row's logit of that class is NaN or +inf. In a whole tile, in the last one, and beside offsets."""
    need_gpu()
    print("logprobs one logit", dtype, rows, dim, classes, value, flush=True)
    lib = handle(dtype)
    for at in (5, classes - 1):
        for masked in (0.0, 0.2):
            c = make(dtype, rows, dim, classes, 8, masked=masked)
            c["x"][:, 0] = 1.0
            c["w"][at, 0] = value
            if masked:
                c["off"][at] = 0.5
            c["y"][:] = 1
            c["y"][2] = at
            out = forward(lib, c, rows, dim, classes, 4)
            for k in ("logprob", "entropy", "lse"):
                assert torch.isnan(out[k]).all(), (k, at, masked)
            ids = out["top_ids"]
            assert ((ids >= -1) & (ids < classes)).all()
            if masked:  # as a masked class it is a constant, whatever its weights hold
                c["off"][at], c["off"][1] = -math.inf, 0.0
                out = forward(lib, c, rows, dim, classes, 4)
                for k in ("entropy", "lse"):
                    assert torch.isfinite(out[k]).all(), (k, at)
                assert out["logprob"][2] == -math.inf and not torch.isnan(out["logprob"]).any() and (out["top_ids"] != at).all()
