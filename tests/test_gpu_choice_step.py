"""Learning from recorded choices with the calls as they are used together: gather -> cross stack -> log probabilities and entropies
-> a policy gradient -> backward -> embedding backward -> Muon on the matrices, AdamW on the rest; eager and as one graph."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import need_gpu, relerr
from paper_2402_06859_amd import rdcn
from paper_2402_06859_amd.step import DeviceAdamW, DeviceBatch, DeviceChoices, DeviceMuon
from paper_2402_06859_amd.synth import WORKLOADS, make_inputs
from test_gpu_logprobs import reference
from test_gpu_softmax_loss import held

pytestmark = pytest.mark.gpu


def build(name="small", batch=200, classes=2003, keep=True, max_norm=None, master=True, parts=True):
    wl = WORKLOADS[name].with_(batch=batch, num_layers=2)
    db = DeviceBatch(wl, make_inputs(wl, bias_std=0.1))
    g = torch.Generator().manual_seed(3)
    dt = torch.bfloat16 if wl.dtype == "bf16" else torch.float32
    w = (torch.randn(classes, wl.d, generator=g) * 0.02).to(dt).cuda()
    labels = torch.randint(0, classes, (batch,), generator=g)
    labels[5:9] = -1
    offset = torch.randn(classes, generator=g)
    offset[classes - 7:] = -float("inf")
    labels.clamp_(max=classes - 8)
    dc = DeviceChoices(db.lib, w, labels.cuda(), offset=offset.cuda(), logit_scale=0.5, top=4, keep=keep)
    old = (torch.randn(batch, generator=g) * 0.2 - 7.5).cuda()          # log probabilities when the choices were made
    advantage = torch.randn(batch, generator=g).cuda()

    def upstream(logprob, entropy):
        # loss = -mean(advantage exp(logprob - old)) - 0.01 mean(entropy)
        ratio = torch.exp(logprob - old)
        return -advantage * ratio / batch, torch.full_like(entropy, -0.01 / batch)

    matrices = []
    for p, g_ in list(zip(db.w_down, db.g_w_down)) + list(zip(db.u, db.g_u)):
        r = wl.rank if parts and p.shape[0] % wl.rank == 0 and p.shape[1] == wl.d else p.shape[0]
        matrices += [(p[i:i + r], g_[i:i + r]) for i in range(0, p.shape[0], r)]   # value, query and key maps apart
    rest = list(zip(db.bias, db.g_bias)) + [(db.q_tables, db.grad_q), (db.r_tables, db.grad_r)] + dc.trained()
    opts = (DeviceMuon(db.lib, matrices, lr=2e-3, weight_decay=0.01, max_norm=max_norm, master=master),
            DeviceAdamW(db.lib, rest, lr=1e-3, max_norm=max_norm, master=master))
    return wl, db, dc, upstream, opts


def state(db, dc, opts):
    out = [dc.logprob, dc.entropy, dc.top_ids, dc.top_logprob, dc.grad_x, dc.grad_w, db.grad_x0] + [g for _, g in db.trained()]
    for opt in opts:
        out += [opt.steps, opt.norm]
        for t in opt.tensors:
            out += [t[k] for k in ("param", "master", "m", "v", "exps") if t.get(k) is not None]
    return out


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("name", ["small", "tiny"])
@pytest.mark.parametrize("keep", [True, False])
def test_gradients_of_a_step(name, keep):
    need_gpu()
    wl, db, dc, upstream, opts = build(name, batch=96, keep=keep)
    W = [p.float().cpu().numpy().astype(np.float64) for p, _ in db.trained()]
    L = wl.num_layers
    dc.train_step(db, upstream)
    torch.cuda.synchronize()
    g, h = upstream(dc.logprob, dc.entropy)
    c = dict(x=db.x_out, w=dc.w, y=dc.labels, off=dc.offset, s=0.5, g=g, h=h)
    ref, bound = reference(c, dc.B, dc.dim, dc.classes, wl.dtype == "f32", 4)
    for k in ("logprob", "entropy", "lse", "top_logprob", "grad_x", "grad_w"):
        held(k, getattr(dc, k), ref[k], bound[k])
    assert torch.equal(dc.top_ids, ref["top_ids"])
    # the stack's gradients for that grad_x, as the library's other tests bound them
    x0 = db.x0.float().cpu().numpy().astype(np.float64)
    gx0, gW, gU, gb = oracle.backward(x0, W[:L], W[L:2 * L], W[2 * L:3 * L], dc.grad_x.float().cpu().numpy().astype(np.float64),
                                      wl.alpha, wl.beta, wl.temperature)
    tol = 5e-2 if wl.dtype == "bf16" else 1e-4
    assert relerr(db.grad_x0.cpu().numpy(), gx0) <= tol
    for l in range(L):
        assert relerr(db.g_w_down[l].cpu().numpy(), gW[l]) <= tol and relerr(db.g_u[l].cpu().numpy(), gU[l]) <= tol
    before = [t["param"].clone() for opt in opts for t in opt.tensors]
    for opt in opts:
        opt.update()
    torch.cuda.synchronize()
    after = [t["param"] for opt in opts for t in opt.tensors]
    assert all(torch.isfinite(p.float()).all() for p in after) and not same(before, after)
    assert db.lib.check_device_errors() == rdcn.RDCN_OK


@pytest.mark.parametrize("opt", [dict(), dict(max_norm=0.01, master=False), dict(name="tiny", keep=False)])
def test_captured_steps_are_the_eager_ones(opt):
    need_gpu()
    print("choice step", opt, flush=True)
    _, db, dc, up, opts = build(**opt)
    _, db2, dc2, up2, opts2 = build(**opt)
    start = [x.clone() for x in state(db, dc, opts)]
    dc.train_step(db, up, opts)  # warm-up outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dc.train_step(db, up, opts)
    for x, s in zip(state(db, dc, opts), start):
        x.copy_(s)
    side = torch.cuda.Stream()
    for i in range(4):
        if i == 2:
            for o in opts + opts2:
                o.set_lr(5e-4)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        dc2.train_step(db2, up2, opts2, side if i % 2 else None)  # eager work between the replays
        torch.cuda.synchronize()
        assert same(state(db, dc, opts), state(db2, dc2, opts2)), "replay %d" % i
    assert [int(o.steps) for o in opts] == [4, 4]


def test_gradients_that_are_not_finite_change_nothing():
    need_gpu()
    _, db, dc, up, opts = build(max_norm=1.0)
    dc.train_step(db, up, opts)
    before = [t[k].clone() for o in opts for t in o.tensors for k in ("param", "m")]
    db.g_w_down[0][3, 5] = float("nan")
    dc.grad_w[0, 0] = float("inf")
    for o in opts:
        o.update()
    torch.cuda.synchronize()
    assert same(before, [t[k] for o in opts for t in o.tensors for k in ("param", "m")])
