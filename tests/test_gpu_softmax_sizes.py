"""Softmax loss at the ends of the sizes it accepts: what a grid cannot hold is refused before anything is launched, what is
accepted runs. (A launch takes less than 2^32 threads along a dimension.)"""
import ctypes
import random

import pytest
import torch

from gpu_helpers import GemmPlan, gemm_plan, need_gpu
from paper_2402_06859_amd import rdcn
from test_gpu_softmax_loss import call_forward, call_grad_within, handle, held, make, reference

pytestmark = pytest.mark.gpu


def workspace(lib, rows, dim, classes):
    s = [ctypes.c_size_t() for _ in range(3)]
    return rdcn.load().rdcn_softmax_loss_workspace(lib.h, rows, dim, classes, *[ctypes.byref(x) for x in s])


def threads(M, N, p, bf16):
    return -(-M // p.bm) * -(-N // p.bn) * (512 if bf16 and p.bm == 256 else 256)


def test_sizes_past_a_grid_are_refused():
    need_gpu()
    OK, S = rdcn.RDCN_OK, rdcn.RDCN_ERR_UNSUPPORTED
    f, b = handle("f32"), handle("bf16")
    K = 1 << 10
    assert workspace(f, 64 * K, 8, K * K - 64) == OK and workspace(f, 64 * K, 8, K * K) == S
    assert workspace(f, 128 * K, 8, K * K) == S and workspace(f, 1, 8, 128 * K * K) == OK
    assert workspace(b, K * K, 8, 128 * K) == OK and workspace(b, K * K, 8, 256 * K) == OK
    assert workspace(b, K * K, 8, K * K) == S                     # blocks of 512 threads, 2^24 of them
    assert workspace(b, 128 * K, 8, 2 * K * K - 128) == OK and workspace(b, 128 * K, 8, 2 * K * K) == S
    assert workspace(b, 16 * K * K, 8, 64) == OK and workspace(f, 16 * K * K, 8, 64) == OK
    assert workspace(f, 64 * K, K * K, 8) == S and workspace(f, 64 * K - 64, K * K, 8) == OK
    assert workspace(b, 8, K * K, 128 * K) == S and workspace(b, 8, K * K, 128 * K - 128) == OK
    assert workspace(b, 8, K * K, 128 * K * K) == S


def test_accepted_sizes_have_grids():
    """Every launch's threads along x, for sizes over the whole range that the library accepts, and the largest of them."""
    need_gpu()
    rng = random.Random(5)
    L = rdcn.load()
    long_plan = L._ZN4rdcn14plan_gemm_longElllb
    long_plan.restype, long_plan.argtypes = GemmPlan, [ctypes.c_int64] * 3 + [ctypes.c_bool]
    libs = {dt: handle(dt) for dt in ("bf16", "f32")}
    span = lambda most: min(most, int(2 ** rng.uniform(0, most.bit_length())))
    seen = 0
    for _ in range(20000):
        dt = rng.choice(("bf16", "f32"))
        bf16 = dt == "bf16"
        rows, dim, classes = span(1 << 24), 8 * span(1 << 17), span(1 << 27)
        if workspace(libs[dt], rows, dim, classes) != rdcn.RDCN_OK:
            # not more than that is refused
            assert max(rows * classes, rows * dim, classes * dim) > 2 ** 35
            continue
        if bf16:
            p = gemm_plan(rows, classes, dim)
            if p.bm == 256 and rows <= 128:
                p.bm = p.bn = 128
        else:
            p = GemmPlan(64, 64, 1, 0, 0)
        assert threads(rows, classes, p, bf16) < 2 ** 32
        for n in (1, 1000, 1024, 1 << 16, 1 << 20, classes):
            n = min(n, classes)
            assert threads(rows, dim, long_plan(rows, dim, n, bf16), bf16) < 2 ** 32
            assert threads(n, dim, long_plan(n, dim, rows, bf16), bf16) < 2 ** 32
        seen += 1
    assert seen > 5000


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_most_rows(dtype):
    """2^24 rows of few classes: a workgroup for each row would be 2^32 threads."""
    need_gpu()
    rows, dim, classes = 1 << 24, 8, 40
    print("softmax loss", dtype, rows, classes, flush=True)
    lib = handle(dtype)
    c = make(dtype, rows, dim, classes, 6, ignored=0.1)
    most = lib.softmax_loss_workspace(rows, dim, classes)[1]
    loss, lse, gx, gw = call_grad_within(lib, c, rows, dim, classes, most)
    total = torch.zeros(classes, dim, dtype=torch.float64, device="cuda")
    bound_w = torch.zeros_like(total)
    part = 1 << 20
    for at in range(0, rows, part):
        ref, bound = reference(dict(c, x=c["x"][at:at + part], y=c["y"][at:at + part]), part, dim, classes, dtype == "f32")
        held("loss", loss[at:at + part], ref[0], bound[0])
        live = c["y"][at:at + part] >= 0
        held("lse", lse[at:at + part][live], ref[1][live], bound[1][live])
        held("grad_x", gx[at:at + part], ref[2], bound[2])
        total += ref[3]
        bound_w += bound[3]
    # (the parts' bounds have a chain of 2^18 additions each; the whole sum's is 16 times that, in the same relative terms)
    held("grad_w", gw, total, 16 * bound_w)


@pytest.mark.parametrize("rows", [5, 200])
def test_more_classes_than_the_large_blocks_offsets_take(rows):
    """Past 1.5 M classes the logits' product keeps the loop that checks its offsets block by block."""
    need_gpu()
    dim, classes = 8 if rows == 5 else 64, 1_700_003
    print("softmax loss", rows, classes, flush=True)
    lib = handle("bf16")
    c = make("bf16", rows, dim, classes, 8, ignored=0.1, masked=0.1)
    c["y"][0], c["y"][1] = classes - 1, classes - 2
    c["off"][classes - 2:] = 0.25
    ref, bound = reference(c, rows, dim, classes, False)
    live = c["y"] >= 0
    loss, lse = call_forward(lib, c, rows, dim, classes)
    held("loss", loss, ref[0], bound[0])
    held("lse", lse[live], ref[1][live], bound[1][live])
    _, most, least = lib.softmax_loss_workspace(rows, dim, classes)
    for size in (most, least):
        got = call_grad_within(lib, c, rows, dim, classes, size)
        for k, name in enumerate(("loss", "lse", "grad_x", "grad_w")):
            at = live if k == 1 else slice(None)
            held("%s, %d bytes" % (name, size), got[k][at], ref[k][at], bound[k][at])
