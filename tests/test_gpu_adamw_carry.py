"""8-bit moments whose blocks' exponents follow a rounding past their last code (RDCN_ROUND_CHANCE_CARRY).

Without it the largest elements of a block stand still at that code: a moving average takes steps of 1 - beta of itself, and
leaves the binade only by one step across the last eighth of it. With it every code is the neighbour above or below with the
probability that keeps the mean, so a moment's mean over many elements is its float one."""
import ctypes
import math

import numpy as np
import pytest
import torch

import test_gpu_adamw as base
from gpu_helpers import need_gpu
from paper_2402_06859_amd import rdcn
from paper_2402_06859_amd.step import DeviceAdamW

pytestmark = pytest.mark.gpu


def encode(x, top, rnd):
    """base.encode with the block's exponent one higher where a code would be past `top`."""
    bits = x.view(np.uint32).astype(np.int64)
    size = bits & 0x7FFFFFFF
    blocks = -(-x.size // 256)
    pad = lambda a: np.pad(a, (0, blocks * 256 - x.size)).reshape(blocks, 256).max(1)
    exps = pad(size) >> 23
    raw = (size + rnd.astype(np.int64)) >> 20
    raw = np.where(size == 0, 0, raw)
    past = pad(np.maximum(raw - base.bases(exps, top).repeat(256)[:x.size], 0)) > top
    exps = exps + (past & (exps < 254))
    code = np.clip(raw - base.bases(exps, top).repeat(256)[:x.size], 0, top)
    if top == 255:
        code = np.maximum(code, 1)
    code = np.where(size == 0, 0, code)
    if top == 127:
        code |= (bits >> 31) << 7
    return code.astype(np.uint8), exps.astype(np.uint8)


@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("master", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
def test_steps_are_the_documented_bits(param, grad, monkeypatch):
    need_gpu()
    print("adamw carry", param, grad, flush=True)
    lib = base.handle()
    went_up = 0

    def counted(x, top, rnd):
        nonlocal went_up
        got, plain = encode(x, top, rnd), old(x, top, rnd)
        went_up += int((got[1] != plain[1]).sum())
        return got

    old = base.encode
    monkeypatch.setattr(base, "encode", counted)
    host, dev, keep = base.make(base.SIZES, param, grad, "8bit", 3)
    lst = rdcn.adamw_tensors(dev)
    for step in range(1, 7):
        lib.adamw_step(lst, step=step, stochastic=True, carry=True, seed=step * 977, **base.HYPER)
        for i, t in enumerate(host):
            base.step32(t, i, base.HYPER, step, 1.0, True, step * 977)
        base.same_state(host, dev, keep)
    assert went_up > 100  # (9% of the blocks hold a largest element past 1.875 of its binade)


def test_moments_at_the_ends_of_the_exponents(monkeypatch):
    """Blocks of every size that a float has: where codes count from 0, and up to the last binade, past which there is none."""
    need_gpu()
    lib = base.handle()
    n = 256 * 254
    rng = np.random.default_rng(7)
    m = np.ldexp(np.where(rng.random(n) < 0.5, -1, 1) * (1.0 + rng.random(n)), (np.arange(n) // 256) - 126).astype(np.float32)
    m.reshape(-1, 256)[:, 0] = np.abs(m.reshape(-1, 256)[:, 0]).view(np.uint32).__or__(0x7FFFFF).view(np.float32)  # ends of binades
    monkeypatch.setattr(base, "encode", encode)
    host, dev, keep = base.make([n], "f32", "f32", "8bit", 3, wd=0.0)
    # moments of that size from a gradient of that size and no decay of the old ones (0)
    with np.errstate(over="ignore"):
        host[0]["grad"] = m / np.float32(0.5)
    host[0]["grad"][~np.isfinite(host[0]["grad"])] = 0
    dev[0]["grad"].copy_(torch.from_numpy(host[0]["grad"]))
    hyper = dict(lr=0.0, beta1=0.5, beta2=0.999, eps=1e-8)
    lib.adamw_step(rdcn.adamw_tensors(dev), step=1, stochastic=True, carry=True, seed=5, **hyper)
    g = dev[0]["grad"].cpu().numpy()
    mm = g * np.float32(0.5)
    h = base.hashed(n, 0, 5)
    cm, em = encode(mm, 127, h >> np.uint32(12))
    assert (dev[0]["m"].cpu().numpy() == cm).all() and (dev[0]["exps"].cpu().numpy()[:n // 256] == em).all()
    back = lib.adamw_values(dev[0]["m"], dev[0]["exps"][:n // 256], True).double().cpu().numpy()
    assert np.isfinite(back).all()
    block = np.abs(mm.astype(np.float64)).reshape(-1, 256).max(1).repeat(256)
    width = np.abs(mm.astype(np.float64)) * 2.0 ** -3 * (1 + 2.0 ** -20) + block * 2.0 ** -14
    assert (np.abs(back - mm) <= np.maximum(width, np.ldexp(1.0, -126))).all()


@pytest.mark.parametrize("kind", ["one size", "sizes", "normal"])
def test_moments_keep_their_mean(kind):
    """1500 updates with gradients of steady size, from DeviceAdamW as it comes. m and v are unbiased, and the elements'
    roundings draw for themselves: the relative noise of one element is at most about 0.25 (an eighth up or down, in a moving average that
    forgets), so the mean of 2^16 of them is within 0.01 of 1 by ten standard deviations. (Without the carry:
    v 0.04 and m 0.94 for one size, v 0.59 for normal gradients.)"""
    need_gpu()
    lib = base.handle()
    n = 1 << 16
    gen = torch.Generator(device="cuda").manual_seed(3)
    size = torch.exp2(torch.randn(n, generator=gen, device="cuda")) if kind == "sizes" else torch.ones(n, device="cuda")
    p, g = torch.zeros(n, device="cuda"), size.clone()
    opt = DeviceAdamW(lib, [(p, g)], lr=0.0, moments="8bit")
    m, v = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for _ in range(1500):
        if kind == "normal":
            g.normal_(generator=gen)
        opt.update()
        m.mul_(0.9).add_(g.double(), alpha=0.1)
        v.mul_(0.999).add_(g.double().square(), alpha=0.001)
    t = opt.tensors[0]
    half = t["exps"].numel() // 2
    got_v = lib.adamw_values(t["v"], t["exps"][half:], False).double()
    got_m = lib.adamw_values(t["m"], t["exps"][:half], True).double()
    assert abs(float((got_v / v).mean()) - 1) < 0.01
    if kind != "normal":  # (normal m are of either sign around 0)
        assert abs(float((got_m / m).mean()) - 1) < 0.01


def test_roundings_that_are_taken():
    need_gpu()
    L = rdcn.load()
    lib = base.handle()
    t = {k: torch.zeros(512, device="cuda") for k in ("param", "grad", "m", "v")}
    lst = rdcn.adamw_tensors([t])
    for value, want in ((0, rdcn.RDCN_OK), (1, rdcn.RDCN_OK), (2, rdcn.RDCN_ERR_ARG), (3, rdcn.RDCN_OK), (4, rdcn.RDCN_ERR_ARG),
                        (-1, rdcn.RDCN_ERR_ARG)):
        c = rdcn.RdcnAdamwConfig(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, None, None, None, value, 0)
        assert L.rdcn_adamw_step(lib.h, ctypes.byref(c), lst, 1, None) == want
    with pytest.raises(rdcn.RdcnError):
        lib.adamw_step(lst, lr=1e-3, carry=True)  # a carry goes with rounding by chance
    torch.cuda.synchronize()
