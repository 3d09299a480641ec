"""Log probabilities with entropy and the most probable classes (rdcn_logprobs_forward), and their gradient
(rdcn_logprobs_grad), against their definition in 64 bits.

Tolerances, derived from the operations (u = 2^-24, half a step of a float), with m the largest logit, d = z - m, rest = the
sum of exp(d) over all classes but that one, and tau = sum p d:
  dz      error of a logit: the chain of at most dim / 4 + 16 additions that the matrix instructions make (bf16 products are
          exact, float ones rounded: dim more), the scale, the offset, their sum: (dim / 4 + 20 [+ dim]) u times the largest
          sum of |x| |w| s + |offset| of the row.
  e(d)    relative error of an exponential: 2 dz for its argument, |d| 2^-23 + 2^-21 for the base-2 unit and the product with
          log2 e, and the sums: one chain over a lane's 32 values, 5 exchanges, the tiles of a row and their joins' factors (an expf
          and three operations each), (tiles / 256 + 64) 8 u.
  log1p   e's mean over the terms of rest, at most sum exp(d) e / (1 + rest), and 2 u of itself.
  logprob log1p's error, and 2 dz + u |d| for the label's own d unless it is the largest by more than 4 dz (then both are the same
          number), and 2 u of the result.
  tau     terms exp(d) |d| (e + 2 u) + exp(d) 2 dz, divided by 1 + rest, and tau times log1p's error.
  lse     dz, log1p's error and 2 u of itself.
  gradient  an element p (-g - h (d - tau)): relative e for p, h times the errors of d (2 dz + u |d|) and tau, half a step of bf16
          (2^-8) for bf16 models, of f16 (2^-11) for p and, by its logarithm, for d where the exponentials are kept, and 2^-40 of
          the row's largest for those that f16 cannot hold, then the products' chains as in the softmax loss's test, and one rounding at the end.
All terms beside these are of second order; every bound is taken 1 + 2^-4 times.
"""
import ctypes
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn
from test_gpu_softmax_loss import DT, U, handle, held, make

pytestmark = pytest.mark.gpu


def upstream(c, rows, seed, entropy=True, logprob=True):
    g = torch.Generator().manual_seed(seed)
    a, b = torch.randn(rows, generator=g) / rows, torch.randn(rows, generator=g) * 0.3 / rows
    if rows > 4:
        a[2], b[2] = 0.0, 0.0
        a[3], b[4] = 0.0, 0.0
    c["g"] = a.cuda() if logprob else None
    c["h"] = b.cuda() if entropy else None
    return c


def buffer(n, fill=0xFF):
    return torch.full((max(n, 256),), fill, dtype=torch.uint8, device="cuda")  # NaN where something reads what nobody wrote


def forward(lib, c, rows, dim, classes, top=0, keep=False, stream=None):
    need = lib.logprobs_workspace(rows, dim, classes, top)
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    out = dict(logprob=f(rows), entropy=f(rows), lse=f(rows), stats=f(rows, 4), kept=buffer(need[1]) if keep else None,
               top_ids=torch.full((rows, top), 77, dtype=c["y"].dtype if c["y"] is not None else torch.int64, device="cuda"),
               top_logprob=f(rows, top))
    if c["y"] is None:
        out["logprob"] = None
    lib.logprobs_forward(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], out["logprob"], out["entropy"],
                         out["lse"], buffer(need[0]), top=top, top_ids=out["top_ids"] if top else None,
                         top_logprob=out["top_logprob"] if top else None, stats=out["stats"], kept=out["kept"], stream=stream)
    return out


def grad(lib, c, rows, dim, classes, out, size=None, stream=None):
    need = lib.logprobs_workspace(rows, dim, classes, 0)
    gx, gw = torch.full_like(c["x"], 7.0), torch.full_like(c["w"], 7.0)
    size = need[2] if size is None else size
    sc = buffer(size + 256)
    lib.logprobs_grad(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], out["stats"], c["g"], c["h"], gx, gw,
                      sc[:max(size, 256)], kept=out["kept"], stream=stream)
    assert (sc[max(size, 256):] == 0xFF).all()
    return gx, gw


def reference(c, rows, dim, classes, f32, top=0):
    """Values and bounds, both in 64 bits: dicts by name."""
    x, w = c["x"].double(), c["w"].double()
    y = torch.full((rows,), -1, device="cuda") if c["y"] is None else c["y"].long()
    kept = (y >= 0) & (y < classes)
    off = torch.zeros(classes, dtype=torch.float64, device="cuda") if c["off"] is None else c["off"].double()
    z = c["s"] * (x @ w.t().contiguous()) + off
    m = z.amax(1, keepdim=True)
    none = torch.isneginf(m)
    d = torch.where(none, -math.inf, z - torch.where(none, 0.0, m))
    ex = torch.exp(d)
    best = z.argmax(1, keepdim=True)
    rest = ex.scatter(1, best, 0.0).sum(1)
    seen = torch.where(torch.isneginf(d), 0.0, d)
    tau = (ex * seen).sum(1) / (1 + rest)
    log_all = torch.log1p(rest)
    at = y.clamp(0, classes - 1)[:, None]
    dy = d.gather(1, at)[:, 0]
    ref = dict(logprob=torch.where(kept, dy - log_all, 0.0), entropy=torch.where(none[:, 0], 0.0, log_all - tau),
               lse=torch.where(none, m, m + log_all[:, None])[:, 0])
    xa, wa = torch.nan_to_num(x, posinf=0.0, neginf=0.0).abs(), w.abs()
    size = c["s"] * (xa @ wa.t().contiguous()).amax(1) + torch.nan_to_num(off, neginf=0.0).abs().max()
    dz = (dim / 4 + 20 + (dim if f32 else 0)) * U * size
    two = 2 * dz[:, None]
    e = torch.exp(two) - 1 + seen.abs() * 2 * 2 * U + 2.0 ** -21 + (classes / 16 / 256 + 64) * 8 * U
    others = ex.scatter(1, best, 0.0)
    dlog = (others * e).sum(1) / (1 + rest) + 2 * U * log_all + 1e-37
    lead = -torch.where(torch.arange(classes, device="cuda") == best, -math.inf, d).amax(1) if classes > 1 else dz * 0 + 1e9
    near = torch.where(lead > 4 * dz, 0.0, 2 * dz)  # how far two largest logits may be confused
    ddy = torch.where((at == best)[:, 0], near, 2 * dz + U * torch.nan_to_num(dy, neginf=0.0).abs())
    dtau = (others * (seen.abs() * (e + 2 * U) + two)).sum(1) / (1 + rest) + tau.abs() * dlog + near
    more = 1 + 2.0 ** -4
    bound = dict(logprob=more * (dlog + ddy + 2 * U * torch.nan_to_num(ref["logprob"], neginf=0.0).abs()),
                 entropy=more * (dlog + dtau + 2 * U * ref["entropy"].abs()),
                 lse=more * (dz + dlog + 2 * U * torch.nan_to_num(ref["lse"], neginf=0.0).abs()))
    if top:
        n = min(top, classes)
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        v, i = v[:, :n], i[:, :n]
        i = torch.where(torch.isneginf(v), -1, i)
        lp = torch.where(torch.isneginf(v), v, v - torch.where(none, 0.0, m) - log_all[:, None])
        pad = (0, top - n)
        ref["top_ids"] = torch.nn.functional.pad(i, pad, value=-1)
        ref["top_logprob"] = torch.nn.functional.pad(lp, pad, value=-math.inf)
        size_lp = torch.nan_to_num(ref["top_logprob"], neginf=0.0).abs()
        bound["top_logprob"] = more * (dlog[:, None] + near[:, None] + 3 * U * size_lp)
    if "g" in c:
        zero = torch.zeros(rows, dtype=torch.float64, device="cuda")
        live = (kept if c["y"] is not None else ~kept) & ~none[:, 0]
        g = torch.where(live & kept, c["g"].double(), zero) if c["g"] is not None else zero
        h = torch.where(live, c["h"].double(), zero) if c["h"] is not None else zero
        live = live & ((g != 0) | (h != 0))
        xk = torch.where(live[:, None], x, 0.0)
        p = ex / (1 + rest)[:, None]
        hot = torch.zeros_like(p).scatter_(1, at, (kept & ~torch.isinf(dy)).double()[:, None])
        g, h, mean = g[:, None], h[:, None], tau[:, None]
        G = c["s"] * torch.where(live[:, None], g * (hot - p) - h * p * (seen - mean), 0.0)
        # the label's own share: 1 - p = (rest, or rest + 1 - exp(d)) / (1 + rest)
        Ga = p * (g.abs() * (1 - hot) + h.abs() * (seen.abs() + mean.abs())) + hot * g.abs() * (1 - p)
        ep = e + dlog[:, None] + 8 * U
        loose = p * h.abs() * (two + U * seen.abs() + dtau[:, None]) + hot * p * g.abs() * torch.maximum(near, ddy)[:, None]
        if f32:
            chain_x, chain_w, r = (classes / 4 + 40) * 2 * U, (rows / 4 + 40) * 2 * U, U
        else:
            chain_x, chain_w, r = (classes / 4 + 40) * U, (rows / 4 + 40) * U, 2.0 ** -8
            ep = (1 + ep) * (1 + 2.0 ** -11) * (1 + 2.0 ** -8) - 1
            loose = loose + p * h.abs() * 2.0 ** -10
        least = torch.where(live[:, None], (g.abs() + h.abs() * 30) * p.amax(1, keepdim=True) * 2.0 ** -40, 0.0) if not f32 else 0.0
        spread = c["s"] * more
        of_live = lambda t: torch.where(live[:, None], spread * t, 0.0)  # (other rows may hold anything)
        bx = of_live(Ga * (ep + chain_x) + loose * (1 + 2.0 ** -7) + least) @ wa
        bw = of_live(Ga * (ep + chain_w) + loose * (1 + 2.0 ** -7) + least).t().contiguous() @ xk.abs()
        ref["grad_x"], ref["grad_w"] = G @ w, G.t().contiguous() @ xk
        bound["grad_x"] = bx * (1 + r) + r * ref["grad_x"].abs() + 1e-37
        bound["grad_w"] = bw * (1 + r) + r * ref["grad_w"].abs() + 1e-37
    return ref, bound


def check(lib, c, rows, dim, classes, f32, top=0, size=None, rows_of=None):
    """Both ways of the gradient: with what the forward kept, and with the logits computed again."""
    ref, bound = reference(c, rows, dim, classes, f32, top)
    pick = slice(None) if rows_of is None else rows_of
    for keep in (False, True):
        out = forward(lib, c, rows, dim, classes, top, keep)
        torch.cuda.synchronize()
        for k in ("logprob", "entropy", "lse") + (("top_logprob",) if top else ()):
            if out[k] is not None:
                held(k, out[k][pick], ref[k][pick], bound[k][pick])
        if top:
            assert torch.equal(out["top_ids"][pick].long(), ref["top_ids"][pick])
        if "g" in c:
            out["grad_x"], out["grad_w"] = grad(lib, c, rows, dim, classes, out, size)
            torch.cuda.synchronize()
            held("grad_x", out["grad_x"], ref["grad_x"], bound["grad_x"])
            held("grad_w", out["grad_w"], ref["grad_w"], bound["grad_w"])
    return out


SIZES = [(1, 8, 1, 1), (1, 8, 3, 2), (2, 16, 8, 8), (1, 64, 1000, 32), (7, 136, 9, 20), (9, 24, 4097, 5), (33, 72, 257, 3),
         (50, 1856, 1003, 8), (64, 512, 4096, 1), (129, 160, 2049, 32), (257, 264, 777, 4), (300, 512, 8197, 7),
         (1000, 64, 33, 10), (1025, 8, 40, 2), (2000, 256, 5003, 8), (5, 4352, 130, 6), (4096, 64, 4, 4), (1024, 1024, 2700, 5),
         (4096, 1024, 2000, 8), (2000, 1024, 20003, 12), (40, 1856, 40001, 8), (3, 512, 70001, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes,top", SIZES)
def test_matches_definition(dtype, rows, dim, classes, top):
    need_gpu()
    print("logprobs", dtype, rows, dim, classes, top, flush=True)
    lib = handle(dtype)
    c = upstream(make(dtype, rows, dim, classes, 13 * rows + classes), rows, 5)
    check(lib, c, rows, dim, classes, dtype == "f32", top)
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype,id_type", [("bf16", "i64"), ("bf16", "i32"), ("f32", "i32")])
@pytest.mark.parametrize("rows,dim,classes", [(5, 40, 65), (70, 72, 515), (333, 136, 1001), (520, 264, 4099)])
def test_masks_and_padding_rows(dtype, id_type, rows, dim, classes):
    need_gpu()
    print("logprobs masks", dtype, id_type, rows, dim, classes, flush=True)
    lib = handle(dtype, id_type)
    c = upstream(make(dtype, rows, dim, classes, 6, ignored=0.4, masked=0.3, id_type=id_type), rows, 7)
    c["y"][-1], c["y"][0], c["y"][2] = -7, -1, 3
    c["x"][c["y"] < 0] = math.nan          # padding rows may hold anything
    c["x"][-1] = math.inf
    c["x"][2] = -math.inf                  # and so may rows whose upstream gradients are 0
    pad = c["y"] < 0
    out = check(lib, c, rows, dim, classes, dtype == "f32", 6, rows_of=torch.nonzero(~pad & torch.isfinite(c["x"][:, 0].float()))[:, 0])
    assert (out["logprob"][pad] == 0).all()
    assert (out["grad_x"][pad] == 0).all() and (out["grad_x"][2] == 0).all()
    assert (out["grad_w"][torch.isneginf(c["off"])] == 0).all()
    ids = out["top_ids"].long()
    assert ((ids >= -1) & (ids < classes)).all()
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_labels_masked_rows_and_lists_longer_than_what_is_visible(dtype):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 20, 32, 300
    c = upstream(make(dtype, rows, dim, classes, 9, masked=0.5), rows, 1)
    c["off"][17], c["y"][3], c["off"][18] = -math.inf, 17, 0.0
    c["g"][3] = 0.5
    out = check(lib, c, rows, dim, classes, dtype == "f32", 8)
    assert out["logprob"][3] == -math.inf and torch.isfinite(out["grad_x"].float()).all()
    c["off"][:] = -math.inf
    c["off"][[250, 3, 77]] = 0.5
    out = check(lib, c, rows, dim, classes, dtype == "f32", 8)
    assert (out["top_ids"][:, 3:] == -1).all() and torch.isneginf(out["top_logprob"][:, 3:]).all()
    c["off"][:] = -math.inf
    c["off"][250] = 0.5                    # one class has all of the probability (a masked label's row keeps the gradient of -lse)
    c["y"][:] = 250
    out = check(lib, c, rows, dim, classes, dtype == "f32", 2)
    assert (out["entropy"] == 0).all() and (out["top_logprob"][:, 0] == 0).all() and (out["grad_x"] == 0).all()
    c["off"][:] = -math.inf
    out = check(lib, c, rows, dim, classes, dtype == "f32", 8)
    assert torch.isneginf(out["logprob"]).all() and torch.isneginf(out["lse"]).all() and (out["entropy"] == 0).all()
    assert (out["top_ids"] == -1).all() and (out["grad_x"] == 0).all() and (out["grad_w"] == 0).all()
    c["off"][:] = torch.finfo(torch.float32).min  # the type's lowest value is a number
    out = forward(lib, c, rows, dim, classes, 8)
    assert torch.isfinite(out["logprob"]).all() and torch.isfinite(out["entropy"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", [(1, 16, 5000), (60, 64, 1003), (300, 64, 9000), (4096, 1024, 2000)])
def test_equal_logits_go_to_the_lowest_class(dtype, rows, dim, classes):
    """All classes alike, and classes that share their weights with many others."""
    need_gpu()
    print("logprobs ties", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 2)
    for top in (1, 7, 32):
        want = torch.arange(top, device="cuda").expand(rows, top)
        x = c["x"].clone()
        c["x"].zero_()
        assert torch.equal(forward(lib, c, rows, dim, classes, top)["top_ids"], want)
        c["x"].copy_(x)
        same = dict(c, w=c["w"][torch.arange(classes, device="cuda") % 37].contiguous())
        z = (same["x"].double() @ same["w"][:37].double().t().contiguous())
        order = torch.sort(z, dim=1, descending=True, stable=True).indices
        reach = -(-(classes - order) // 37)  # how many classes are equal to each
        got = forward(lib, same, rows, dim, classes, top)["top_ids"]
        first = order[:, :1] + 37 * torch.arange(top, device="cuda")
        assert (reach[:, 0] >= 27).all()
        n = min(top, 27)
        assert torch.equal(got[:, :n], first[:, :n])
    for row in (0, rows - 1):   # two equal ones at the border of a list
        c["x"][row] = 0
        c["x"][row, 0] = 1
    c["w"][:, 0] = 0
    c["w"][classes - 1, 0] = c["w"][5, 0] = c["w"][321, 0] = 2
    ids = forward(lib, c, rows, dim, classes, 2)["top_ids"]
    assert ids[0].tolist() == [5, 321] and ids[-1].tolist() == [5, 321]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_with_all_their_probability_on_one_class_keep_their_digits(dtype):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 16, 64, 4096
    c = upstream(make(dtype, rows, dim, classes, 3), rows, 3)
    for n in range(rows):
        c["x"][n] = 0
        c["x"][n, n] = 8.0
        c["w"][:, n] = 0
        c["w"][c["y"][n], n] = 1.5 + 0.25 * n
    out = check(lib, c, rows, dim, classes, dtype == "f32", 4)
    ref, bound = reference(c, rows, dim, classes, dtype == "f32", 4)
    assert float(ref["entropy"].min()) < 1e-7 and (bound["entropy"] < 1e-3 * ref["entropy"]).all()
    assert (out["entropy"] > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_far_apart_and_large(dtype):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 40, 64, 1000
    c = upstream(make(dtype, rows, dim, classes, 13, sharp=60.0), rows, 2)
    check(lib, c, rows, dim, classes, dtype == "f32", 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["logprob", "entropy", "no labels"])
def test_one_upstream_gradient_alone(dtype, which):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 90, 72, 700
    c = upstream(make(dtype, rows, dim, classes, 8, ignored=0.2), rows, 4, entropy=which != "logprob", logprob=which == "logprob")
    if which == "no labels":
        c["y"] = None
    out = check(lib, c, rows, dim, classes, dtype == "f32", 3)
    assert (out["grad_w"] != 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_label_past_the_classes_is_reported_and_left_out(dtype):
    need_gpu()
    lib = handle(dtype)
    for rows, dim, classes in ((5, 16, 13), (200, 72, 515)):
        c = upstream(make(dtype, rows, dim, classes, 4), rows, 4)
        c["g"][:] = 1.0
        c["y"][2], c["y"][4] = classes, 1 << 40
        out = check(lib, c, rows, dim, classes, dtype == "f32")
        assert lib.check_device_errors() == rdcn.RDCN_ERR_INDEX
        assert lib.check_device_errors() == rdcn.RDCN_OK
        assert out["logprob"][2] == 0 and (out["grad_x"][2] == 0).all() and out["logprob"][4] == 0


@pytest.mark.parametrize("dtype,rows,dim,classes", [("bf16", 300, 264, 5003), ("f32", 130, 68, 3075), ("bf16", 2000, 64, 9000),
                                                    ("bf16", 1100, 512, 33001), ("bf16", 20, 136, 9001), ("bf16", 32, 1024, 5003),
                                                    ("bf16", 33, 1024, 5003)])
def test_less_scratch_means_pieces_of_the_classes(dtype, rows, dim, classes):
    need_gpu()
    print("logprobs in pieces", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    c = upstream(make(dtype, rows, dim, classes, 21, ignored=0.2, masked=0.1), rows, 6)
    c["y"][7], c["y"][8] = classes - 1, classes - 3
    c["off"][classes - 3:] = 0.25
    most, least = lib.logprobs_workspace(rows, dim, classes, 0)[2:]
    assert least < most
    for size in (least, (least + most) // 2 // 256 * 256, most - 256, most + 4096):
        check(lib, c, rows, dim, classes, dtype == "f32", size=size)


@pytest.mark.parametrize("rows,dim,classes,top", [(1, 8, 8201, 3), (16, 136, 9001, 32), (13, 4352, 8209, 5), (2, 512, 50000, 8),
                                                  (16, 1856, 20003, 8), (17, 512, 20003, 8), (16, 1000, 33001, 8), (64, 512, 50001, 8),
                                                  (17, 72, 31003, 4), (40, 72, 100003, 8), (1, 64, 90113, 32), (64, 1000, 91003, 5)])
def test_few_rows_of_many_classes(rows, dim, classes, top):
    need_gpu()
    print("logprobs of few rows", rows, dim, classes, flush=True)
    lib = handle("bf16")
    c = upstream(make("bf16", rows, dim, classes, 31 * rows, ignored=0.1, masked=0.1), rows, 8)
    c["off"][:70] = -math.inf  # a tile without any class
    c["y"][0] = classes - 1
    c["off"][classes - 1] = 0.5
    most, least = lib.logprobs_workspace(rows, dim, classes, top)[2:]
    for size in (most, least):
        check(lib, c, rows, dim, classes, False, top, size=size)
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype,rows,dim", [("bf16", 2100, 64), ("f32", 2100, 24)])
def test_gradient_where_the_rows_have_a_launch_of_their_own(dtype, rows, dim):
    """More than 2^26 kept exponentials, whole and in pieces, with a label that is out of range."""
    need_gpu()
    classes = 32003
    lib = handle(dtype)
    c = upstream(make(dtype, rows, dim, classes, 23, ignored=0.1, masked=0.1), rows, 7)
    c["y"][5] = classes + 3
    most, least = lib.logprobs_workspace(rows, dim, classes, 0)[2:]
    for size in (most, (most + least) // 2 // 256 * 256):
        check(lib, c, rows, dim, classes, dtype == "f32", size=size)
        assert lib.check_device_errors() == rdcn.RDCN_ERR_INDEX


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(dtype):
    need_gpu()
    lib = handle(dtype)
    c = upstream(make(dtype, 1, 24, 13, 1), 1, 1)
    c = dict(c, x=c["x"][:0], y=c["y"][:0], g=c["g"][:0], h=c["h"][:0])
    out = forward(lib, c, 0, 24, 13, 3)
    gx, gw = grad(lib, c, 0, 24, 13, out)
    assert (gw == 0).all() and gx.numel() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(dtype):
    """Central differences in 64 bits of sum g logprob + h entropy along random directions: their error is of order h^2 (third
    derivatives, for logits that move by up to 1e-4 of their size), far below the elements' bounds added up."""
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 12, 40, 130
    c = upstream(make(dtype, rows, dim, classes, 17, masked=0.1), rows, 9)
    c["off"][c["y"]] = 0.5
    ref, bound = reference(c, rows, dim, classes, dtype == "f32")
    out = forward(lib, c, rows, dim, classes)
    gx, gw = grad(lib, c, rows, dim, classes, out)
    x, w, off = c["x"].double(), c["w"].double(), c["off"].double()

    def loss(x, w):
        lp = torch.log_softmax(c["s"] * (x @ w.t().contiguous()) + off, 1)
        p = lp.exp()
        ent = -(p * lp.masked_fill(torch.isneginf(lp), 0.0)).sum(1)
        return float((c["g"].double() * lp.gather(1, c["y"][:, None])[:, 0] + c["h"].double() * ent).sum())

    gen = torch.Generator().manual_seed(1)
    for _ in range(3):
        vx = torch.randn(rows, dim, generator=gen, dtype=torch.float64).cuda()
        vw = torch.randn(classes, dim, generator=gen, dtype=torch.float64).cuda()
        t = 1e-5
        slope = (loss(x + t * vx, w + t * vw) - loss(x - t * vx, w - t * vw)) / (2 * t)
        got = float((gx.double() * vx).sum() + (gw.double() * vw).sum())
        room = float((bound["grad_x"] * vx.abs()).sum() + (bound["grad_w"] * vw.abs()).sum()) + 1e-7
        assert abs(got - slope) <= room


def test_results_that_are_not_wanted_and_repeated_calls():
    need_gpu()
    lib = handle("bf16")
    rows, dim, classes = 70, 72, 1500
    c = make("bf16", rows, dim, classes, 3)
    full = forward(lib, c, rows, dim, classes, 4)
    again = forward(lib, c, rows, dim, classes, 4)
    for k in ("logprob", "entropy", "lse", "stats", "top_ids", "top_logprob"):
        assert torch.equal(full[k], again[k])
    ids = torch.zeros(rows, 4, dtype=torch.int64, device="cuda")
    sc = buffer(lib.logprobs_workspace(rows, dim, classes, 4)[0])
    lib.logprobs_forward(rows, dim, classes, c["x"], c["w"], None, None, c["s"], None, None, None, sc, top=4, top_ids=ids)
    assert torch.equal(ids, full["top_ids"])


def test_forward_and_gradient_in_a_graph_and_on_another_stream():
    need_gpu()
    lib = handle("bf16")
    rows, dim, classes = 200, 136, 5000
    c = upstream(make("bf16", rows, dim, classes, 12, ignored=0.1), rows, 1)
    need = lib.logprobs_workspace(rows, dim, classes, 6)
    out = dict(logprob=torch.empty(rows, device="cuda"), entropy=torch.empty(rows, device="cuda"),
               lse=torch.empty(rows, device="cuda"), top_ids=torch.empty(rows, 6, dtype=torch.int64, device="cuda"),
               top_logprob=torch.empty(rows, 6, device="cuda"), gx=torch.empty_like(c["x"]), gw=torch.empty_like(c["w"]))
    stats, kept, sc = torch.empty(rows, 4, device="cuda"), buffer(need[1]), buffer(max(need[0], need[2]))

    def both(o, stream=None):
        lib.logprobs_forward(rows, dim, classes, c["x"], c["w"], None, c["y"], c["s"], o["logprob"], o["entropy"], o["lse"], sc,
                             top=6, top_ids=o["top_ids"], top_logprob=o["top_logprob"], stats=stats, kept=kept, stream=stream)
        lib.logprobs_grad(rows, dim, classes, c["x"], c["w"], None, c["y"], c["s"], stats, c["g"], c["h"], o["gx"], o["gw"], sc,
                          kept=kept, stream=stream)

    both(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out)
    x0 = c["x"].clone()
    for i in range(4):
        c["x"].copy_(x0 * (1 + i))
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = {k: torch.zeros_like(v) for k, v in out.items()}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        both(eager, side if i % 2 else None)
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], eager[k]) for k in out), "replay %d" % i


def test_refusals():
    need_gpu()
    lib = handle("bf16")
    rows, dim, classes = 6, 16, 50
    c = upstream(make("bf16", rows, dim, classes, 1), rows, 1)
    need = lib.logprobs_workspace(rows, dim, classes, 3)
    sc = buffer(max(need[0], need[2]) + 256)
    f = torch.zeros(rows, device="cuda")
    stats, ids = torch.zeros(rows, 4, device="cuda"), torch.zeros(rows, 3, dtype=torch.int64, device="cuda")

    def status(call):
        try:
            call()
        except rdcn.RdcnError as err:
            return err.status
        return 0

    def fwd(dim=dim, classes=classes, x=c["x"], w=c["w"], y=c["y"], s=0.5, scratch=sc, lp=f, top=3, ids=ids, **kw):
        return status(lambda: lib.logprobs_forward(rows, dim, classes, x, w, None, y, s, lp, f, f, scratch, top=top, top_ids=ids,
                                                   **kw))

    assert fwd() == 0
    assert fwd(dim=12) == rdcn.RDCN_ERR_UNSUPPORTED
    assert fwd(top=rdcn.LOGPROBS_TOP_MAX + 1, ids=torch.zeros(rows, 40, dtype=torch.int64, device="cuda")) == rdcn.RDCN_ERR_UNSUPPORTED
    assert fwd(top=-1, ids=None) == rdcn.RDCN_ERR_ARG and fwd(ids=None) == rdcn.RDCN_ERR_ARG
    assert fwd(s=math.nan) == rdcn.RDCN_ERR_ARG and fwd(y=None) == rdcn.RDCN_ERR_ARG
    assert fwd(scratch=None) == rdcn.RDCN_ERR_WORKSPACE and fwd(scratch=sc[:max(0, need[0] - 256)]) == rdcn.RDCN_ERR_WORKSPACE
    assert fwd(scratch=sc[8:]) == rdcn.RDCN_ERR_WORKSPACE
    for bad in (dict(x=c["x"].float()), dict(w=c["w"][1:]), dict(y=c["y"].int()), dict(lp=f.double()), dict(ids=ids.int()),
                dict(x=c["x"].t()), dict(stats=stats[:5])):
        with pytest.raises(ValueError):
            fwd(**bad)
    gx, gw = torch.empty_like(c["x"]), torch.empty_like(c["w"])

    def bwd(y=c["y"], g=c["g"], scratch=sc, gx=gx, stats=stats, s=0.5):
        return status(lambda: lib.logprobs_grad(rows, dim, classes, c["x"], c["w"], None, y, s, stats, g, c["h"], gx, gw, scratch))

    assert bwd() == 0
    assert bwd(y=None) == rdcn.RDCN_ERR_ARG and bwd(y=None, g=None) == 0
    assert bwd(stats=None) == rdcn.RDCN_ERR_ARG and bwd(s=math.inf) == rdcn.RDCN_ERR_ARG
    assert bwd(scratch=sc[:max(0, need[3] - 256)]) == rdcn.RDCN_ERR_WORKSPACE
    with pytest.raises(ValueError):
        bwd(gx=gx.float())
    assert lib.check_device_errors() == rdcn.RDCN_OK
