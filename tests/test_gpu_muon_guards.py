"""The Muon step's guards in both kinds of kernels (one workgroup a matrix, and launches of blocks) and in lists that mix sizes.

X's tolerance for five steps, 2e-4 of its norm: as derived in test_gpu_muon_spectra.py.
"""
import math

import pytest
import torch

from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn
from test_gpu_muon import handle, matrix, momentum_of, newton_schulz, only_update, step

pytestmark = pytest.mark.gpu

SMALL, LARGE, MIXED = [(40, 90), (90, 40)], [(130, 200), (200, 130)], [(130, 200), (40, 30), (200, 130), (5, 70)]


def listed(shapes, params=("master", "bf16", "f32"), **kw):
    return [matrix(r, c, i + 1, params[i % len(params)], **kw) for i, (r, c) in enumerate(shapes)]


def state(ts):
    return [t[k] for t in ts for k in ("param", "master", "m") if t.get(k) is not None]


def copies(ts):
    return [{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()} for t in ts]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(state(a), state(b)))


@pytest.mark.parametrize("shapes", [SMALL, LARGE, MIXED])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_clip_factor_that_is_not_finite_changes_nothing(shapes, bad):
    need_gpu()
    lib = handle()
    ts = listed(shapes)
    before = copies(ts)
    clip = torch.tensor([bad], device="cuda")
    step(lib, ts, lr=0.1, clip=clip, stochastic=True)
    assert equal(ts, before)
    clip.fill_(0.25)
    step(lib, ts, lr=0.1, clip=clip)
    step(lib, before, lr=0.1, grad_scale=0.25)
    assert equal(ts, before) and all((t["m"] != 0).any() for t in ts)


@pytest.mark.parametrize("shapes", [SMALL, LARGE, MIXED])
def test_without_a_gradient_the_weights_decay(shapes):
    """And one whose gradient is there, beside them, takes its step."""
    need_gpu()
    lib = handle()
    ts = listed(shapes, ("f32",))
    for t in ts[:-1]:
        t["grad"].zero_()
        t["m"].zero_()
    before = copies(ts)
    step(lib, ts, lr=0.5)
    decay = torch.tensor(1 - 0.5 * 0.02, dtype=torch.float64).float().cuda()
    for t, b in zip(ts[:-1], before):
        assert torch.equal(t["param"], b["param"] * decay) and (t["m"] == 0).all()
    alone = [before[-1]]
    _, u = momentum_of(alone[0], 0.95, True)
    want = alone[0]["param"].double() * (1 - 0.5 * 0.02) - 0.5 * 1.5 * newton_schulz(u)
    # X's tolerance, and a few roundings of the weights
    assert float((ts[-1]["param"].double() - want).norm()) <= 0.75 * 2e-4 * float(newton_schulz(u).norm()) + 2.0 ** -22 * float(want.norm())


@pytest.mark.parametrize("shapes", [SMALL, LARGE, MIXED])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_gradient_that_is_not_finite_reaches_its_own_weights_alone(shapes, bad):
    need_gpu()
    lib = handle()
    for which in range(len(shapes)):
        ts, clean = listed(shapes, ("f32",)), listed(shapes, ("f32",))
        ts[which]["grad"][3, 3] = bad
        step(lib, ts, lr=0.1)
        step(lib, clean, lr=0.1)
        for i, (t, o) in enumerate(zip(ts, clean)):
            if i == which:
                assert torch.isnan(t["param"]).any()
            else:
                assert torch.equal(t["param"], o["param"]) and torch.equal(t["m"], o["m"])


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e18, 1e30])
@pytest.mark.parametrize("rows,cols", [(130, 200), (300, 70)])
def test_the_size_of_a_gradient_does_not_count(rows, cols, size):
    need_gpu()
    lib = handle()
    t = only_update(matrix(rows, cols, 8, falling=False))
    t["grad"] *= size
    t["m"] *= size
    _, u = momentum_of(t, 0.95, True)
    step(lib, [t])
    ref = newton_schulz(u)
    assert float((t["param"].double() - ref).norm()) <= 2e-4 * float(ref.norm())


@pytest.mark.parametrize("shapes", [SMALL, MIXED])
def test_bf16_weights_rounded_by_chance(shapes):
    need_gpu()
    lib = handle()
    ts = listed(shapes, ("bf16",))
    exact = [dict(t, param=t["param"].float(), m=t["m"].clone()) for t in ts]
    step(lib, ts, lr=0.01, stochastic=True, seed=99)
    step(lib, exact, lr=0.01)
    for i, (t, w) in enumerate(zip(ts, exact)):
        h = torch.arange(t["param"].numel(), dtype=torch.int64) ^ ((99 + 0x9E3779B9 * (i + 1)) & 0xFFFFFFFF)
        h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
        h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
        h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
        bits = (w["param"].cpu().view(torch.int32).flatten().long() & 0xFFFFFFFF) + (h >> 16)
        assert torch.equal(t["param"].cpu().view(torch.int16).flatten().long() & 0xFFFF, (bits >> 16) & 0xFFFF)


@pytest.mark.parametrize("shapes", [SMALL, LARGE, MIXED])
def test_captured_steps_are_the_eager_ones(shapes):
    need_gpu()
    lib = handle()
    ts = listed(shapes, ("bf16", "master", "f32"))
    other, start = copies(ts), copies(ts)
    lists = [rdcn.muon_tensors(x) for x in (ts, other)]
    sc = [torch.empty(lib.muon_workspace(lists[0]), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lr, number = torch.tensor([0.01], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    clip = torch.ones(1, device="cuda")

    def one(i):
        lib.muon_step(lists[i], sc[i], lr=0.0, device_lr=lr, device_step=number, clip=clip, stochastic=True, seed=5)

    one(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(0)
    for x, s in zip(state(ts), state(start)):
        x.copy_(s)
    for i in range(4):
        number.fill_(i + 1)
        lr.fill_(0.01 * (i + 1))
        clip.fill_(math.nan if i == 2 else 0.5)  # (a step that is left out, and one behind it)
        before = copies(ts)
        graph.replay()
        one(1)
        torch.cuda.synchronize()
        assert equal(ts, other), "replay %d" % i
        assert equal(ts, before) == (i == 2)
