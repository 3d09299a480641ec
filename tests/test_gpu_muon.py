"""The Muon step (rdcn_muon_step) against its definition in 64 bits.

The update X alone is seen with weights of 0, no decay and lr scale = -1. Its tolerance, relative in the 2-norm of the elements: a
product of pairs drops lo lo (2^-22 of |a| |b|) and rounds two operands to 22 bits (2^-23 each), and its float sums add 2^-24 a step
of which the errors' mean counts: e = 3 * 2^-22 of the operands' norms in all. Between two fresh starts A passes at most three steps, each
of which multiplies an error of it by up to a^2 (11.9), and T = a + b A + c A^2 by |b| (4.8; T is at least 0.6): e * 11.9^2 * 4.8 / 0.6 =
8.1e-4 of X's norm, and less than that again for the few products that follow. So TOL = 1e-3, of the whole and, as errors are spread
evenly, five times that for every 64 x 64 block against the blocks' mean. (A single f16 in place of a pair leaves 3e-3 to 5e-1.)
The momentum is two roundings of float products and their sum: equal to torch's, to the bit.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn

pytestmark = pytest.mark.gpu

ABC = (3.4445, -4.7750, 2.0315)
TOL = 1e-3
U = 2.0 ** -24


def handle():
    return rdcn.Rdcn(rdcn.make_config(64, 4, 16, 32, 8, 1, 25, 25, 600))


def matrix(rows, cols, seed, param="f32", grad="f32", falling=True, **kw):
    g = torch.Generator().manual_seed(seed)
    short = min(rows, cols)

    def make():
        if not falling:
            return torch.randn(rows, cols, generator=g)
        s = torch.arange(1, short + 1, dtype=torch.float32) ** -0.5
        return torch.randn(rows, short, generator=g) * s @ torch.randn(short, cols, generator=g)

    p = torch.randn(rows, cols, generator=g) * 0.05
    t = dict(param=p if param == "f32" else p.bfloat16(), master=p if param == "master" else None,
             grad=make().to(torch.float32 if grad == "f32" else torch.bfloat16), m=make() * 0.3, weight_decay=0.02, scale=1.5)
    t.update(kw)
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in t.items()}


def only_update(t):
    t["param"] = torch.zeros_like(t["param"], dtype=torch.float32)
    t.update(master=None, weight_decay=0.0, scale=-1.0)
    return t


def step(lib, ts, lr=1.0, stream=None, **kw):
    lst = rdcn.muon_tensors(ts)
    need = lib.muon_workspace(lst)
    sc = torch.full((max(need, 256) + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN where something reads what nobody wrote
    lib.muon_step(lst, sc[:max(need, 256)], lr=lr, stream=stream, **kw)
    assert (sc[max(need, 256):] == 0xFF).all()


def momentum_of(t, mu, nesterov, gs=1.0):
    """m' and U in float, each operation one rounding."""
    c1 = torch.tensor(1.0 - mu, dtype=torch.float64).float()
    mu = torch.tensor(mu, dtype=torch.float64).float()
    g = t["grad"].float() * gs
    m = t["m"] * mu.cuda() + g * c1.cuda()
    return m, (m * mu.cuda() + g * c1.cuda() if nesterov else m)


def newton_schulz(u, abc=ABC, steps=5):
    x = u.double().cpu() if u.numel() < 1 << 16 else u.double()
    norm = x.norm()
    x = x / norm if norm > 0 else x
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    a, b, c = abc
    for _ in range(steps):
        q = x @ x.t().contiguous()
        x = a * x + (b * q + c * (q @ q)) @ x
    return (x.t() if tall else x).contiguous().cuda()


def held(got, ref, tol=TOL):
    d = (got.double() - ref)
    norm = float(ref.norm())
    assert float(d.norm()) <= tol * norm, "off by %.3g of the norm" % (float(d.norm()) / max(norm, 1e-300))
    pad = (0, -d.shape[1] % 64, 0, -d.shape[0] % 64)
    blocks = torch.nn.functional.pad(d, pad).unfold(0, 64, 64).unfold(1, 64, 64).double().pow(2).sum((2, 3)).sqrt()
    mean = norm / math.sqrt(blocks.numel())
    assert float(blocks.max()) <= 5 * tol * max(mean, norm / math.sqrt(ref.numel())), "a block off by %.3g" % float(blocks.max() / mean)


SHAPES = [(1, 1), (1, 7), (9, 1), (3, 5), (64, 64), (65, 63), (32, 160), (160, 32), (100, 37), (129, 1000), (1000, 130), (257, 257),
          (333, 1001), (37, 20011), (512, 512), (768, 1856), (1856, 256), (1024, 640), (1500, 1500),
          (64, 1024), (1024, 63), (1, 1024), (64, 1025), (65, 1024)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_update_matches_definition(rows, cols):
    need_gpu()
    print("muon", rows, cols, flush=True)
    lib = handle()
    for falling, nesterov, grad in ((False, True, "f32"), (True, False, "bf16")):
        t = only_update(matrix(rows, cols, rows + 3 * cols, falling=falling, grad=grad))
        m, u = momentum_of(t, 0.95, nesterov)
        step(lib, [t], nesterov=nesterov)
        torch.cuda.synchronize()
        assert torch.equal(t["m"], m)
        held(t["param"], newton_schulz(u))


@pytest.mark.parametrize("shapes", [[(5701, 5733)], [(5733, 5701)], [(4100, 4300), (4500, 4100)]])
def test_more_than_a_round_of_large_blocks(shapes):
    """Whole rounds of 256 x 256 blocks, and what is left of the last matrix in quarters, some of which lie behind its end."""
    need_gpu()
    lib = handle()
    ts = [only_update(matrix(r, c, i, falling=False)) for i, (r, c) in enumerate(shapes)]
    us = [momentum_of(t, 0.95, True) for t in ts]
    step(lib, ts)
    torch.cuda.synchronize()
    for t, (m, u) in zip(ts, us):
        assert torch.equal(t["m"], m)
        held(t["param"], newton_schulz(u))


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 8])
def test_other_numbers_of_steps(steps):
    need_gpu()
    lib = handle()
    for rows, cols in ((70, 200), (200, 90)):
        t = only_update(matrix(rows, cols, 5))
        _, u = momentum_of(t, 0.9, True)
        step(lib, [t], steps=steps, momentum=0.9)
        held(t["param"], newton_schulz(u, steps=steps))


def test_coefficients_that_end_at_one():
    """2, -1.5, 0.5 keeps singular values of 1: after many steps the rows are orthonormal."""
    need_gpu()
    lib = handle()
    abc = (2.0, -1.5, 0.5)
    t = only_update(matrix(60, 300, 3, falling=False))
    _, u = momentum_of(t, 0.95, True)
    step(lib, [t], coefficients=abc, steps=12)
    held(t["param"], newton_schulz(u, abc, 12))
    x = t["param"].double()
    assert float((x @ x.t() - torch.eye(60, dtype=torch.float64, device="cuda")).abs().max()) <= 1e-4


@pytest.mark.parametrize("param", ["f32", "master", "bf16"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_weights_take_the_step(param, grad):
    need_gpu()
    lib = handle()
    lr = 0.01
    for rows, cols in ((96, 264), (101, 43), (320, 128)):
        t = matrix(rows, cols, 9, param, grad)
        p0 = (t["master"] if param == "master" else t["param"]).double()
        m, u = momentum_of(t, 0.95, True, gs=0.5)
        x = newton_schulz(u)
        step(lib, [t], lr=lr, grad_scale=0.5)
        want = p0 * (1 - lr * 0.02) - lr * 1.5 * x
        got = t["master"] if param == "master" else t["param"]
        # decay and its product, size and its product, the difference: one rounding each; X's own error, five times its
        # norm's share for a block, up to six times that for an element
        bound = 4 * U * (p0.abs() + want.abs() + lr * 1.5 * x.abs()) + lr * 1.5 * 30 * TOL * float(x.norm()) / math.sqrt(x.numel())
        if param == "bf16":
            bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        assert ((got.double() - want).abs() <= bound).all()
        assert torch.equal(t["m"], m)
        if param == "master":
            assert torch.equal(t["param"], t["master"].bfloat16())


def test_bf16_weights_rounded_by_chance():
    need_gpu()
    lib = handle()
    a, b = matrix(77, 130, 4, "bf16"), matrix(130, 77, 5, "bf16")
    f = [dict(t, param=t["param"].float(), m=t["m"].clone()) for t in (a, b)]
    step(lib, [a, b], lr=0.01, stochastic=True, seed=99)
    step(lib, f, lr=0.01)
    for i, (t, w) in enumerate(zip((a, b), f)):
        n = t["param"].numel()
        h = torch.arange(n, dtype=torch.int64) ^ ((99 + 0x9E3779B9 * (i + 1)) & 0xFFFFFFFF)
        h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
        h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
        h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
        bits = (w["param"].cpu().view(torch.int32).flatten().long() & 0xFFFFFFFF) + (h >> 16)
        got = t["param"].cpu().view(torch.int16).flatten().long() & 0xFFFF
        assert torch.equal(got, (bits >> 16) & 0xFFFF)


def test_many_matrices_in_one_list():
    """More than one run of launches, matrices of no elements, short ones among them and alone. Which others share a launch may change
    the order of a matrix's sums (each result holds the definition's tolerance), but not its momentum, and a list's results are the same
    bits every time."""
    need_gpu()
    lib = handle()
    shapes = [(33 + 7 * i, 40 + 13 * ((i * 5) % 9)) for i in range(27)] + [(0, 5), (5, 0)]

    def make():
        return [matrix(r, c, i, ("f32", "master")[i % 2], ("f32", "bf16")[i % 3 == 0]) if r * c else
                dict(param=torch.zeros(r, c, device="cuda"), grad=torch.zeros(r, c, device="cuda"), m=torch.zeros(r, c, device="cuda"))
                for i, (r, c) in enumerate(shapes)]

    ts, again, alone = make(), make(), make()
    want = []
    for t in ts:
        if t["param"].numel():
            m, u = momentum_of(t, 0.95, True)
            w = t.get("master")
            want.append((m, (t["param"] if w is None else w).double(), newton_schulz(u)))
        else:
            want.append(None)
    step(lib, ts, lr=0.01)
    step(lib, again, lr=0.01)
    for t, o, one, ref in zip(ts, again, alone, want):
        assert torch.equal(t["param"], o["param"]) and torch.equal(t["m"], o["m"])
        if ref is None:
            continue
        step(lib, [one], lr=0.01)
        m, p0, x = ref
        for got in (t, one):
            assert torch.equal(got["m"], m)
            w = got["param"] if got.get("master") is None else got["master"]
            room = 8 * U * float(p0.norm()) + 0.01 * 1.5 * TOL * float(x.norm())
            assert float((w.double() - (p0 * (1 - 0.01 * 0.02) - 0.01 * 1.5 * x)).norm()) <= room


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1.0, 1e18, 1e30])
def test_the_size_of_a_gradient_does_not_count(size):
    need_gpu()
    lib = handle()
    t = only_update(matrix(50, 120, 8, falling=False))
    t["grad"] *= size
    t["m"] *= size
    _, u = momentum_of(t, 0.95, True)
    step(lib, [t])
    held(t["param"], newton_schulz(u))


def test_one_large_element_and_no_gradient():
    need_gpu()
    lib = handle()
    t = only_update(matrix(500, 700, 8, falling=False))
    t["grad"][3, 5] = 1e6
    _, u = momentum_of(t, 0.95, True)
    step(lib, [t])
    held(t["param"], newton_schulz(u))
    t = matrix(30, 20, 1)
    t["grad"].zero_()
    t["m"].zero_()
    p = t["param"].clone()
    step(lib, [t], lr=0.5)
    assert torch.equal(t["param"], p * torch.tensor(1 - 0.5 * 0.02, dtype=torch.float64).float().cuda())
    assert (t["m"] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_clip_factor_that_is_not_finite_changes_nothing(bad):
    need_gpu()
    lib = handle()
    ts = [matrix(40, 90, 1, "master"), matrix(90, 40, 2, "bf16")]
    before = [t[k].clone() for t in ts for k in ("param", "m")]
    clip = torch.tensor([bad], device="cuda")
    step(lib, ts, lr=0.1, clip=clip, stochastic=True)
    assert all(torch.equal(a, b) for a, b in zip(before, [t[k] for t in ts for k in ("param", "m")]))
    clip.fill_(0.25)
    other = [{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()} for t in ts]
    step(lib, ts, lr=0.1, clip=clip)
    step(lib, other, lr=0.1, grad_scale=0.25)
    assert all(torch.equal(t[k], o[k]) for t, o in zip(ts, other) for k in ("param", "m"))


def test_a_gradient_that_is_not_finite_reaches_its_own_weights_alone():
    need_gpu()
    lib = handle()
    ts = [matrix(40, 90, 1), matrix(90, 40, 2)]
    ts[0]["grad"][3, 3] = math.nan
    step(lib, ts, lr=0.1)
    assert torch.isnan(ts[0]["param"]).any() and torch.isfinite(ts[1]["param"]).all()


def test_captured_steps_are_the_eager_ones():
    need_gpu()
    lib = handle()
    ts = [matrix(48, 160, 1, "bf16"), matrix(160, 48, 2, "master"), matrix(300, 300, 3)]
    other = [{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()} for t in ts]
    lists = [rdcn.muon_tensors(x) for x in (ts, other)]
    sc = [torch.empty(lib.muon_workspace(lists[0]), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lr, number = torch.tensor([0.01], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def one(i, stream=None):
        lib.muon_step(lists[i], sc[i], lr=0.0, device_lr=lr, device_step=number, stochastic=True, seed=5, stream=stream)

    start = [t[k].clone() for t in ts for k in ("param", "m")]
    one(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(0)
    for x, s in zip([t[k] for t in ts for k in ("param", "m")], start):
        x.copy_(s)
    ts[1]["master"].copy_(other[1]["master"])
    for i in range(4):
        number.fill_(i + 1)
        lr.fill_(0.01 * (i + 1))
        graph.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        one(1, side if i % 2 else None)
        torch.cuda.synchronize()
        assert all(torch.equal(t[k], o[k]) for t, o in zip(ts, other) for k in ("param", "m")), "replay %d" % i


def test_refusals():
    need_gpu()
    lib = handle()
    t = matrix(20, 30, 1)
    lst = rdcn.muon_tensors([t])
    sc = torch.empty(lib.muon_workspace(lst), dtype=torch.uint8, device="cuda")

    def status(lst=lst, sc=sc, lr=0.1, **kw):
        try:
            lib.muon_step(lst, sc, lr=lr, **kw)
        except rdcn.RdcnError as err:
            return err.status
        return 0

    assert status() == 0
    A, X, W = rdcn.RDCN_ERR_ARG, rdcn.RDCN_ERR_UNSUPPORTED, rdcn.RDCN_ERR_WORKSPACE
    assert status(lr=math.nan) == A and status(momentum=1.0) == A and status(momentum=-0.1) == A and status(steps=0) == A
    assert status(steps=17) == X and status(grad_scale=math.inf) == A and status(stochastic=2) == A
    assert status(coefficients=(10.0, 0.0, 0.0)) == X and status(coefficients=(math.nan, 0.0, 0.0)) == A
    assert status(sc=None) == W and status(sc=sc[:-256]) == W and status(sc=sc[16:]) == W
    assert status(lst=rdcn.muon_tensors([t, t])) == A
    for field, value in (("param", 8), ("grad", None), ("m", None), ("rows", -1), ("param_dtype", 7), ("grad_dtype", 2),
                         ("scale", math.nan), ("weight_decay", math.inf)):
        bad = rdcn.muon_tensors([t])
        setattr(bad[0], field, value)
        assert status(lst=bad) == A, field
    for rows, cols in ((1 << 21, 4), (1 << 15, 1 << 15)):
        bad = rdcn.muon_tensors([t])
        bad[0].rows, bad[0].cols = rows, cols
        assert status(lst=bad) == X
    bad = rdcn.muon_tensors([t])
    bad[0].master = t["m"].data_ptr()
    assert status(lst=bad) == A
    for bad in (dict(grad=t["grad"][:-1]), dict(m=t["m"].double()), dict(param=t["param"].flatten()), dict(grad=t["grad"].half()),
                dict(m=t["m"].t().contiguous().t()), dict(master=t["param"].clone())):
        with pytest.raises(ValueError):
            rdcn.muon_tensors([dict(t, **bad)])
    assert lib.muon_workspace(rdcn.muon_tensors([])) == 0 and status(lst=rdcn.muon_tensors([]), sc=None) == 0
