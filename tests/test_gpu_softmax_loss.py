"""Softmax loss over many classes (rdcn_softmax_loss_forward / _grad) against its definition in 64 bits.

Tolerances, derived from the operations (u = 2^-24, half a step of a float):
  logits    a float sum of exact products (bf16) or of rounded ones (float): the matrix instructions add at
            least 4 products a time, so a chain has at most dim / 4 + 16 additions, each off by u of the
            partial sum, which is at most A = max over classes of s * sum |x| |w|; the scale, the offset and
            their sum add 3 u (A + |offset|). Float products are rounded too (u A each).
  lse       one logit's error, plus the sums (8 per thread, 5 over lanes, one per tile, logs) and the
            exponentials' relative errors: each at most 2^-21 for arguments down to -87, where a term of
            that size still counts. loss: lse's error and the label's logit's.
  gradients G's elements carry the error of exp(z - lse), at most e = exp(2 dz) - 1 + 2^-21 for dz = the
            error of a logit and of lse, for bf16 models half a step of f16 (2^-11, the exponentials that are
            kept) and of bf16 (2^-8), and the float products' chain as above; then each gradient is
            rounded once. With |G| taken as f (p + onehot), the bound is elementwise. bf16 models keep
            exponentials exp(z - tile's maximum) <= 1 in f16 times 2^15: f16 is spaced by 2^-24 below its
            normal numbers, so half a step is 2^-25 and 2^-25 / 2^15 = 2^-40 of the tile's largest
            exponential, at most 2^-40 of the row's largest p. G gets f times that as an absolute error.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def handle(dtype, id_type="i64"):
    return rdcn.Rdcn(rdcn.make_config(64, 4, 16, 32, 8, 1, 25, 25, 600, dtype=dtype, id_type=id_type))


def make(dtype, rows, dim, classes, seed, ignored=0.0, masked=0.0, weights=False, sharp=2.0, id_type="i64"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, dim, generator=g)
    w = torch.randn(classes, dim, generator=g) * (sharp / math.sqrt(dim))
    y = torch.randint(0, classes, (rows,), generator=g)
    off = None
    if masked is not None and masked > 0:
        off = torch.randn(classes, generator=g)
        off[torch.rand(classes, generator=g) < masked] = -math.inf
    if ignored:
        y[torch.rand(rows, generator=g) < ignored] = -1
    wt = torch.rand(rows, generator=g) + 0.5 if weights else None
    if wt is not None:
        wt[0] = 0.0
    to = lambda t, d=None: None if t is None else (t if d is None else t.to(d)).cuda().contiguous()
    return dict(x=to(x, DT[dtype]), w=to(w, DT[dtype]), y=to(y, torch.int64 if id_type == "i64" else torch.int32),
                off=to(off), wt=to(wt), s=0.75, scale=1.0 / 7)


def call_forward(lib, c, rows, dim, classes, stream=None):
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    sc = torch.empty(max(256, lib.softmax_loss_workspace(rows, dim, classes)[0]), dtype=torch.uint8, device="cuda")
    sc.fill_(0xFF)  # NaN where something reads what nobody wrote
    lib.softmax_loss_forward(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], loss, lse, sc, stream)
    return loss, lse


def call_grad(lib, c, rows, dim, classes, stream=None):
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    gx, gw = torch.full_like(c["x"], 7.0), torch.full_like(c["w"], 7.0)
    sc = torch.empty(max(256, lib.softmax_loss_workspace(rows, dim, classes)[1]), dtype=torch.uint8, device="cuda")
    sc.fill_(0xFF)
    lib.softmax_loss_grad(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], c["wt"], c["scale"], loss, lse,
                          gx, gw, sc, stream)
    return loss, lse, gx, gw


def reference(c, rows, dim, classes, f32):
    """Definition in 64 bits on the device of the inputs, and the elementwise bounds."""
    x, w, y = c["x"].double(), c["w"].double(), c["y"].long()
    kept = (y >= 0) & (y < classes)
    off = torch.zeros(classes, dtype=torch.float64, device=x.device) if c["off"] is None else c["off"].double()
    z = c["s"] * (x @ w.t().contiguous()) + off
    lse = torch.logsumexp(z, 1)
    at = y.clamp(0, classes - 1)[:, None]
    zy = z.gather(1, at)[:, 0]
    loss = torch.where(kept, lse - zy, 0.0)
    loss = torch.where(kept & torch.isinf(zy), math.inf, loss)
    p = torch.where(torch.isneginf(z), 0.0, torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None]))
    hot = torch.zeros_like(p).scatter_(1, at, (kept & ~torch.isinf(zy)).double()[:, None])
    f = kept.double() * c["scale"] * c["s"]
    if c["wt"] is not None:
        f = f * c["wt"].double()
    xk = torch.where(kept[:, None], x, 0.0)
    live = f != 0
    G = torch.where(live[:, None], f[:, None] * (p - hot), 0.0)
    Ga = torch.where(live[:, None], f.abs()[:, None] * (p + hot), 0.0)
    gx, gw = G @ w, G.t().contiguous() @ xk
    xa, wa = torch.nan_to_num(xk).abs(), w.abs()
    size = c["s"] * (xa @ wa.t().contiguous()).amax(1) + torch.nan_to_num(off, neginf=0.0).abs().max()
    dz = (dim / 4 + 20 + (dim if f32 else 0)) * U * size
    dl = dz + (classes / 256 + 64) * U + 2.0 ** -21 + U * torch.nan_to_num(lse, neginf=0.0).abs()
    dloss = dl + dz + 2 * U * torch.nan_to_num(loss, posinf=0.0)
    e = torch.exp(dz + dl) - 1 + 2.0 ** -21
    if f32:
        chain_x, chain_w, r, eg = (classes / 4 + 40) * 2 * U, (rows / 4 + 40) * 2 * U, U, e + 4 * U
    else:
        chain_x, chain_w, r = (classes / 4 + 40) * U, (rows / 4 + 40) * U, 2.0 ** -8
        eg = (1 + e) * (1 + 2.0 ** -11) * (1 + 2.0 ** -8) - 1
    # floats' smallest steps: products of values this small need not keep relative digits
    tiny = 1e-37
    least = torch.zeros_like(f) if f32 else torch.where(live, f.abs() * p.amax(1) * 2.0 ** -40 * (1 + 2.0 ** -7), 0.0)
    bx = (Ga * (eg[:, None] + chain_x) + least[:, None]) @ wa
    bw = (Ga * (eg[:, None] + chain_w) + least[:, None]).t().contiguous() @ xa
    return (loss, lse, gx, gw), (dloss, dl, bx + r * gx.abs() + r * bx + tiny, bw + r * gw.abs() + r * bw + tiny)


def held(name, got, ref, bound):
    got, ref = got.double(), ref.double()
    same = got == ref  # infinities
    bad = ~same & ~((got - ref).abs() <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %.3g over a bound of %.3g" % (
        name, int(bad.sum()), bad.numel(), float((got - ref).abs()[bad].max()), float(bound[bad].min()))


def check(lib, c, rows, dim, classes, f32):
    ref, bound = reference(c, rows, dim, classes, f32)
    kept = (c["y"] >= 0) & (c["y"] < classes)
    loss, lse = call_forward(lib, c, rows, dim, classes)
    got = call_grad(lib, c, rows, dim, classes)
    torch.cuda.synchronize()
    for tag, (lo, ls) in (("forward", (loss, lse)), ("grad", got[:2])):
        held(tag + " loss", lo, ref[0], bound[0])
        held(tag + " lse", ls[kept], ref[1][kept], bound[1][kept])
    held("grad_x", got[2], ref[2], bound[2])
    held("grad_w", got[3], ref[3], bound[3])
    return got


SIZES = [(1, 8, 1), (1, 8, 3), (2, 16, 8), (1, 64, 1000), (7, 136, 9), (9, 24, 4097), (33, 72, 257), (50, 1856, 1003),
         (64, 512, 4096), (129, 160, 2049), (257, 264, 777), (300, 512, 8197), (1000, 64, 33), (1025, 8, 40),
         (2000, 256, 5003), (5, 4352, 130), (4096, 64, 4), (600, 1024, 9000),
         (1024, 1024, 2700), (4096, 1024, 2000), (2000, 1024, 20003), (40, 1856, 40001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", SIZES)
def test_matches_definition(dtype, rows, dim, classes):
    need_gpu()
    print("softmax loss", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 11 * rows + classes)
    check(lib, c, rows, dim, classes, dtype == "f32")
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", [(5, 1024, 4000), (5, 2048, 4200), (1, 8, 20000), (700, 64, 70), (3, 1600, 64)])
def test_few_and_many_small_blocks(dtype, rows, dim, classes):
    """Gradients whose products go in one launch (up to 2048 blocks together) and those that take one each; with one of
    them much the larger, and with one split along its sum and the other not."""
    need_gpu()
    print("softmax loss blocks", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 29, ignored=0.1, masked=0.1, weights=True)
    check(lib, c, rows, dim, classes, dtype == "f32")
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype,id_type", [("bf16", "i64"), ("bf16", "i32"), ("f32", "i32")])
@pytest.mark.parametrize("rows,dim,classes", [(3, 40, 65), (70, 72, 515), (333, 136, 1001), (520, 264, 4099)])
def test_masks_padding_rows_and_weights(dtype, id_type, rows, dim, classes):
    need_gpu()
    print("softmax loss masks", dtype, id_type, rows, dim, classes, flush=True)
    lib = handle(dtype, id_type)
    c = make(dtype, rows, dim, classes, 5, ignored=0.4, masked=0.3, weights=True, id_type=id_type)
    c["y"][-1] = -7
    c["x"][c["y"] < 0] = math.nan          # padding rows may hold anything
    c["x"][-1] = math.inf
    c["x"][0] = -math.inf                  # a row of weight 0 too (its loss is what its x makes of it)
    c["y"][0] = -1
    got = check(lib, c, rows, dim, classes, dtype == "f32")
    pad = c["y"] < 0
    assert (got[0][pad] == 0).all() and (got[2][pad] == 0).all()
    assert (got[3][torch.isneginf(c["off"])] == 0).all()
    assert lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,classes", [(20, 32, 300), (300, 64, 9000)])
def test_rows_of_weight_zero_add_nothing(dtype, rows, dim, classes):
    need_gpu()
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 19, weights=True)
    clean = call_grad(lib, c, rows, dim, classes)
    c["wt"][7] = 0.0
    c["x"][0], c["x"][7] = math.nan, math.inf
    got = call_grad(lib, c, rows, dim, classes)
    assert (got[2][0] == 0).all() and (got[2][7] == 0).all() and torch.isfinite(got[3].float()).all()
    c["x"][0], c["x"][7] = 0.0, 0.0
    assert torch.equal(call_grad(lib, c, rows, dim, classes)[3], got[3])
    assert torch.equal(clean[2][1:7], got[2][1:7])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_label_or_every_class_is_masked(dtype):
    need_gpu()
    lib = handle(dtype)
    rows, dim, classes = 20, 32, 300
    c = make(dtype, rows, dim, classes, 9, masked=0.5)
    c["off"][17] = -math.inf
    c["y"][3] = 17
    c["off"][18] = 0.0
    got = check(lib, c, rows, dim, classes, dtype == "f32")
    assert got[0][3] == math.inf and torch.isfinite(got[2].float()).all()
    c["off"][:] = -math.inf
    got = check(lib, c, rows, dim, classes, dtype == "f32")
    assert (got[0] == math.inf).all() and torch.isneginf(got[1]).all()
    assert (got[2] == 0).all() and (got[3] == 0).all()
    c["off"][:] = torch.finfo(torch.float32).min  # the type's lowest value is a number: it cancels
    lo, ls = call_forward(lib, c, rows, dim, classes)
    assert torch.isfinite(lo).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_label_past_the_classes_is_reported_and_left_out(dtype):
    need_gpu()
    lib = handle(dtype)
    for rows, dim, classes in ((5, 16, 13), (200, 72, 515)):
        c = make(dtype, rows, dim, classes, 4)
        c["y"][2] = classes            # in the padding of the last column group
        c["y"][4] = 1 << 40
        got = check(lib, c, rows, dim, classes, dtype == "f32")
        assert lib.check_device_errors() == rdcn.RDCN_ERR_INDEX
        assert lib.check_device_errors() == rdcn.RDCN_OK
        assert got[0][2] == 0 and (got[2][2] == 0).all() and got[0][4] == 0


def call_grad_within(lib, c, rows, dim, classes, size):
    """call_grad with a scratch of that size, and 256 bytes behind it that stay as they are."""
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    gx, gw = torch.full_like(c["x"], 7.0), torch.full_like(c["w"], 7.0)
    sc = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    lib.softmax_loss_grad(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], c["wt"], c["scale"], loss, lse,
                          gx, gw, sc[:size])
    assert (sc[size:] == 0xFF).all()
    return loss, lse, gx, gw


@pytest.mark.parametrize("dtype,rows,dim,classes", [("bf16", 300, 264, 5003), ("f32", 130, 68, 3075), ("bf16", 2000, 64, 9000),
                                                    ("bf16", 1100, 512, 33001), ("bf16", 4096, 1024, 4099),
                                                    ("bf16", 1280, 1024, 4100)])
def test_less_scratch_means_pieces_of_the_classes(dtype, rows, dim, classes):
    need_gpu()
    print("softmax loss in pieces", dtype, rows, dim, classes, flush=True)
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 21, ignored=0.2, masked=0.1, weights=True)
    c["y"][7], c["y"][8] = classes - 1, classes - 3
    c["off"][classes - 3:] = 0.25
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    assert least < most
    ref, bound = reference(c, rows, dim, classes, dtype == "f32")
    # pieces add their sums in float: one more rounding of the running sum for each (counted in `chain`)
    for size in (least, (least + most) // 2 // 256 * 256, most - 256, most, most + 4096):
        got = call_grad_within(lib, c, rows, dim, classes, size)
        for k, name in enumerate(("loss", "lse", "grad_x", "grad_w")):
            live = (c["y"] >= 0) if k == 1 else slice(None)
            held("%s with %d bytes" % (name, size), got[k][live], ref[k][live], bound[k][live])


def test_a_gradient_in_the_logits_too_large_to_ask_for_whole():
    """Past 4 GiB the workspace asks for pieces by itself: 17000 x 131077 in bf16."""
    need_gpu()
    rows, dim, classes = 17000, 8, 131077
    print("softmax loss", rows, classes, flush=True)
    lib = handle("bf16")
    most = lib.softmax_loss_workspace(rows, dim, classes)[1]
    assert most < 3 << 30
    c = make("bf16", rows, dim, classes, 22, ignored=0.2)
    got = call_grad_within(lib, c, rows, dim, classes, most)
    # a stretch of rows against the definition (the sums over all rows: against another size of scratch)
    part = dict(c, x=c["x"][16000:16500], y=c["y"][16000:16500])
    ref, bound = reference(part, 500, dim, classes, False)
    held("loss", got[0][16000:16500], ref[0], bound[0])
    held("grad_x", got[2][16000:16500], ref[2], bound[2])
    other = call_grad_within(lib, c, rows, dim, classes, most // 2)
    # both are within half a step of bf16 of sums that differ by their order: 2^-7 and the chains' roundings
    scale = got[3].float().abs() * 2.0 ** -7 + 1e-6 * got[3].float().abs().max()
    assert ((got[3].float() - other[3].float()).abs() <= scale).all()


def test_sharp_rows_keep_the_digits_of_one_minus_p():
    """A label of probability close to 1: its gradient f (p - 1) is small and must not be p's rounding error."""
    need_gpu()
    lib = handle("bf16")
    rows, dim, classes = 16, 64, 4096
    c = make("bf16", rows, dim, classes, 3)
    for n in range(rows):
        c["x"][n] = 0
        c["x"][n, n] = 8.0
        c["w"][:, n] = 0
        c["w"][c["y"][n], n] = 2.75
    ref, bound = reference(c, rows, dim, classes, False)
    p = torch.exp(-ref[0])
    assert (p > 0.99).any()
    check(lib, c, rows, dim, classes, False)


def test_logits_far_apart_and_large():
    need_gpu()
    lib = handle("f32")
    rows, dim, classes = 40, 64, 1000
    c = make("f32", rows, dim, classes, 13, sharp=60.0)
    check(lib, c, rows, dim, classes, True)
    lib = handle("bf16")
    c = make("bf16", rows, dim, classes, 13, sharp=60.0)
    check(lib, c, rows, dim, classes, False)


def test_no_rows():
    need_gpu()
    for dtype in ("bf16", "f32"):
        lib = handle(dtype)
        c = make(dtype, 1, 24, 13, 1)
        got = call_grad(lib, dict(c, x=c["x"][:0], y=c["y"][:0]), 0, 24, 13)
        assert (got[3] == 0).all() and got[2].numel() == 0
        call_forward(lib, dict(c, x=c["x"][:0], y=c["y"][:0]), 0, 24, 13)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_against_differences(dtype):
    """Central differences of the loss in 64 bits along random directions: their own error is of
    order h^2 (third derivatives of a loss whose logits move by at most 1e-3 h-steps), the bound of
    the gradient's elements is added up along the direction."""
    need_gpu()
    rows, dim, classes = 30, 40, 203
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 17, ignored=0.2, masked=0.2, weights=True)
    _, bound = reference(c, rows, dim, classes, dtype == "f32")
    _, _, gx, gw = call_grad(lib, c, rows, dim, classes)

    def total(x, w):
        z = c["s"] * (x @ w.t().contiguous()) + c["off"].double()
        kept = c["y"] >= 0
        l = torch.logsumexp(z, 1) - z.gather(1, c["y"].clamp(min=0)[:, None])[:, 0]
        fine = kept & torch.isfinite(l)
        lse = torch.logsumexp(z, 1)
        l = torch.where(kept & ~fine, lse, torch.where(fine, l, 0.0))  # a masked label: the gradient of lse
        return float((l * c["wt"].double()).sum() * c["scale"])

    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, h = c["x"].double(), c["w"].double(), 1e-5
    for _ in range(4):
        dx = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        dw = torch.randn(w.shape, generator=g, device="cuda", dtype=torch.float64)
        num = (total(x + h * dx, w + h * dw) - total(x - h * dx, w - h * dw)) / (2 * h)
        got = float((gx.double() * dx).sum() + (gw.double() * dw).sum())
        tol = float((bound[2] * dx.abs()).sum() + (bound[3] * dw.abs()).sum())
        assert abs(num - got) <= tol + 1e-6 * abs(num) + 1e-7


def test_offsets_past_32_bits():
    """w of more than 2^31 values: the last classes' logits are read from the right place."""
    need_gpu()
    lib = handle("bf16")
    rows, dim, classes = 3, 16384, 140003
    print("softmax loss, w of", classes * dim, "values", flush=True)
    w = torch.zeros(classes, dim, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    w[-70:] = torch.randn(70, dim, generator=g, device="cuda").bfloat16() * 0.01
    x = torch.randn(rows, dim, generator=g, device="cuda").bfloat16()
    y = torch.tensor([classes - 1, classes - 66, 5], device="cuda")
    c = dict(x=x, w=w, y=y, off=None, wt=None, s=1.0, scale=1.0)
    z = torch.zeros(rows, classes, dtype=torch.float64, device="cuda")
    z[:, -70:] = x.double() @ w[-70:].double().t().contiguous()
    lse = torch.logsumexp(z, 1)
    ref = lse - z.gather(1, y[:, None])[:, 0]
    size = (x.double().abs() @ w[-70:].double().abs().t().contiguous()).amax(1)
    tol = 2 * (dim / 4 + 20) * U * size + (classes / 64 + 64) * U + 2.0 ** -20 + 4 * U * lse
    loss, got = call_forward(lib, c, rows, dim, classes)
    assert ((got.double() - lse).abs() <= tol).all() and ((loss.double() - ref).abs() <= tol).all()
    out = call_grad(lib, c, rows, dim, classes)
    assert ((out[0].double() - ref).abs() <= tol).all()
    p = torch.softmax(z, 1)
    p[torch.arange(3), y] -= 1
    ref_w = p[:, -70:].t().contiguous() @ x.double()
    ref_a = p[:, -70:].abs().t().contiguous() @ x.double().abs()
    held("grad_w", out[3][-70:], ref_w, ref_a * (2.0 ** -7) + ref_w.abs() * 2.0 ** -8 + 1e-30)


def test_replays_and_other_streams_give_the_same_bits():
    need_gpu()
    lib = handle("bf16")
    for rows, dim, classes in ((333, 136, 1001), (900, 512, 6000)):
        c = make("bf16", rows, dim, classes, 31, ignored=0.2, masked=0.1)
        want = call_grad(lib, c, rows, dim, classes)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = call_grad(lib, c, rows, dim, classes)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        gx, gw = torch.empty_like(c["x"]), torch.empty_like(c["w"])
        sc = torch.empty(lib.softmax_loss_workspace(rows, dim, classes)[1], dtype=torch.uint8, device="cuda")

        def step():
            lib.softmax_loss_grad(rows, dim, classes, c["x"], c["w"], c["off"], c["y"], c["s"], None, c["scale"], loss,
                                  lse, gx, gw, sc)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            for t in (loss, lse, gx, gw):
                t.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, gx, gw)))
            call_grad(lib, c, rows, dim, classes)  # eager work between the replays
        x0 = c["x"].clone()
        c["x"].copy_(c["x"].flip(0))               # the same graph on new values
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(call_grad(lib, c, rows, dim, classes), (loss, lse, gx, gw)))
        c["x"].copy_(x0)


def test_refusals():
    need_gpu()
    L = rdcn.load()
    lib = handle("bf16")
    c = make("bf16", 4, 16, 10, 1)
    loss, lse = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    gx, gw = torch.empty_like(c["x"]), torch.empty_like(c["w"])
    need = lib.softmax_loss_workspace(4, 16, 10)
    sc = torch.empty(need[1] + 256, dtype=torch.uint8, device="cuda")
    P = lambda t: None if t is None else t.data_ptr()

    def fwd(rows=4, dim=16, classes=10, x=c["x"], w=c["w"], y=c["y"], s=1.0, lo=loss, ls=lse, scr=P(sc), n=need[1], xo=0):
        return L.rdcn_softmax_loss_forward(lib.h, rows, dim, classes, None if x is None else P(x) + xo, P(w), None, P(y),
                                           s, P(lo), P(ls), scr, n, None)

    def grad(scale=1.0, a=gx, b=gw, scr=P(sc), n=need[1], s=1.0):
        return L.rdcn_softmax_loss_grad(lib.h, 4, 16, 10, P(c["x"]), P(c["w"]), None, P(c["y"]), s, None, scale, P(loss),
                                        P(lse), P(a), P(b), scr, n, None)

    A, S, W = rdcn.RDCN_ERR_ARG, rdcn.RDCN_ERR_UNSUPPORTED, rdcn.RDCN_ERR_WORKSPACE
    assert fwd(rows=-1) == A and fwd(dim=0) == A and fwd(classes=0) == A
    assert fwd(dim=12) == S and fwd(rows=(1 << 24) + 1) == S and fwd(classes=(1 << 27) + 1) == S
    assert fwd(rows=1 << 24, classes=1 << 27) == S
    assert fwd(x=None) == A and fwd(w=None) == A and fwd(y=None) == A and fwd(lo=None) == A and fwd(ls=None) == A
    assert fwd(s=math.nan) == A and fwd(xo=2) == A
    assert fwd(scr=None) == W and fwd(scr=P(sc) + 16) == W and fwd(n=need[0] - 1) == W
    assert grad(scale=math.inf) == A and grad(s=math.inf) == A and grad(scale=1e30, s=1e30) == A and grad(a=None) == A and grad(b=None) == A
    assert grad(n=need[2] - 1) == W and grad(scr=None) == W and grad(scr=P(sc) + 128) == W
    assert fwd() == rdcn.RDCN_OK and grad() == rdcn.RDCN_OK
    torch.cuda.synchronize()
