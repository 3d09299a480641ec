"""The log probability and Muon calls: struct layouts, and refusals that need no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2402_06859_amd import rdcn
from paper_2402_06859_amd.step import DeviceChoices

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_c(tmp_path):
    prog = tmp_path / "mlayout.c"
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rdcn.h"\n'
                    'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu %zu %d\\n", sizeof(rdcn_muon_tensor),'
                    ' offsetof(rdcn_muon_tensor, rows), offsetof(rdcn_muon_tensor, scale),'
                    ' offsetof(rdcn_muon_tensor, grad_dtype), sizeof(rdcn_muon_config), offsetof(rdcn_muon_config, steps),'
                    ' offsetof(rdcn_muon_config, clip), offsetof(rdcn_muon_config, seed), RDCN_LOGPROBS_TOP_MAX); return 0;}\n')
    exe = tmp_path / "mlayout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    vals = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    T, C = rdcn.RdcnMuonTensor, rdcn.RdcnMuonConfig
    assert vals == [ctypes.sizeof(T), T.rows.offset, T.scale.offset, T.grad_dtype.offset, ctypes.sizeof(C), C.steps.offset,
                    C.clip.offset, C.seed.offset, rdcn.LOGPROBS_TOP_MAX]


def test_null_handles_are_refused():
    L = rdcn.load()
    s = [ctypes.c_size_t() for _ in range(4)]
    r = [ctypes.byref(x) for x in s]
    A = rdcn.RDCN_ERR_ARG
    assert L.rdcn_logprobs_workspace(None, 1, 8, 8, 0, *r) == A
    assert L.rdcn_logprobs_forward(None, 1, 8, 8, None, None, None, None, 1.0, 0, None, None, None, None, None, None, None, 0,
                                   None, 0, None) == A
    assert L.rdcn_logprobs_grad(None, 1, 8, 8, None, None, None, None, 1.0, None, None, 0, None, None, None, None, None, 0,
                                None) == A
    c = rdcn.RdcnMuonConfig(1e-3, 0.95, 1.0, 2.0, -1.5, 0.5, 5, 1, None, None, None, 0, 0)
    lst = (rdcn.RdcnMuonTensor * 1)()
    assert L.rdcn_muon_workspace(None, lst, 1, r[0]) == A
    assert L.rdcn_muon_step(None, ctypes.byref(c), lst, 1, None, 0, None) == A


def test_descriptors_check_their_tensors():
    def t(**kw):
        d = {k: torch.zeros(20, 30) for k in ("param", "grad", "m")}
        d.update(kw)
        return d

    bf = torch.zeros(20, 30, dtype=torch.bfloat16)
    lst = rdcn.muon_tensors([t(), t(param=bf, master=torch.zeros(20, 30), grad=bf, scale=2.0, weight_decay=0.5)])
    assert [(x.rows, x.cols) for x in lst] == [(20, 30)] * 2 and [x.param_dtype for x in lst] == [0, 1]
    assert lst[1].scale == 2.0 and lst[1].weight_decay == 0.5 and lst[0].scale == 1.0 and lst[0].master is None
    for bad in (t(param=torch.zeros(600), grad=torch.zeros(600), m=torch.zeros(600)), t(grad=torch.zeros(30, 20)),
                t(m=torch.zeros(20, 30, dtype=torch.float64)), t(m=bf), t(param=torch.zeros(20, 60)[:, ::2]),
                t(grad=torch.zeros(20, 30, dtype=torch.float16)), t(master=torch.zeros(20, 30)),
                t(param=torch.zeros(20, 30, dtype=torch.int32))):
        with pytest.raises(ValueError):
            rdcn.muon_tensors([bad])


class Recorder:
    """Stands where a handle would: what fits reaches it."""

    def __init__(self, dtype=rdcn.BF16, id_type=rdcn.I64):
        self.cfg = rdcn.RdcnConfig(dtype=dtype, id_type=id_type)
        self.h = None

    _choices = rdcn.Rdcn._choices
    logprobs_forward = rdcn.Rdcn.logprobs_forward
    logprobs_grad = rdcn.Rdcn.logprobs_grad


def test_the_binding_refuses_tensors_that_the_kernels_would_read_past():
    rows, dim, classes = 5, 16, 40
    x, w = torch.zeros(rows, dim, dtype=torch.bfloat16), torch.zeros(classes, dim, dtype=torch.bfloat16)
    y, f = torch.zeros(rows, dtype=torch.int64), torch.zeros(rows)
    ids, lp, st = torch.zeros(rows, 3, dtype=torch.int64), torch.zeros(rows, 3), torch.zeros(rows, 4)
    sc = torch.zeros(256, dtype=torch.uint8)
    good = dict(x=x, w=w, offset=torch.zeros(classes), labels=y, logit_scale=1.0, logprob=f, entropy=f, lse=f, scratch=sc, top=3,
                top_ids=ids, top_logprob=lp, stats=st)
    r = Recorder()
    for name, bad in (("x", x[:4]), ("x", x.float()), ("w", w[:, :8]), ("w", w.t()), ("offset", torch.zeros(classes - 1)),
                      ("offset", torch.zeros(classes).double()), ("labels", y.int()), ("labels", y[:4]), ("logprob", f[:4]),
                      ("entropy", f.bfloat16()), ("lse", torch.zeros(2 * rows)[::2]), ("top_ids", ids.int()), ("top_ids", ids[:, :2]),
                      ("top_logprob", lp[:4]), ("stats", st[:4])):
        with pytest.raises(ValueError, match=name):
            r.logprobs_forward(rows, dim, classes, **dict(good, **{name: bad}))
    grad = dict(x=x, w=w, offset=None, labels=y, logit_scale=1.0, stats=st, grad_logprob=f, grad_entropy=f,
                grad_x=torch.zeros_like(x), grad_w=torch.zeros_like(w), scratch=sc)
    for name, bad in (("grad_logprob", f[:4]), ("grad_entropy", f.double()), ("grad_x", x.float()), ("grad_w", w[:39]),
                      ("stats", st[:, :3])):
        with pytest.raises(ValueError, match=name):
            r.logprobs_grad(rows, dim, classes, **dict(grad, **{name: bad}))


def test_device_choices_checks_devices():
    with pytest.raises(ValueError):
        DeviceChoices(Recorder(), torch.zeros(40, 16, dtype=torch.bfloat16, device="meta"), torch.zeros(5, dtype=torch.int64))
