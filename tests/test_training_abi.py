"""The training calls (softmax loss, AdamW, gradient norm): struct layouts, and refusals that need no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2402_06859_amd import rdcn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_adamw_struct_layouts_match_c(tmp_path):
    prog = tmp_path / "alayout.c"
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rdcn.h"\n'
                    'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu\\n", sizeof(rdcn_adamw_tensor),'
                    ' offsetof(rdcn_adamw_tensor, n), offsetof(rdcn_adamw_tensor, moments), sizeof(rdcn_adamw_config),'
                    ' offsetof(rdcn_adamw_config, step), offsetof(rdcn_adamw_config, clip),'
                    ' offsetof(rdcn_adamw_config, seed)); return 0;}\n')
    exe = tmp_path / "alayout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    vals = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    T, C = rdcn.RdcnAdamwTensor, rdcn.RdcnAdamwConfig
    assert vals == [ctypes.sizeof(T), T.n.offset, T.moments.offset, ctypes.sizeof(C), C.step.offset, C.clip.offset,
                    C.seed.offset]


def test_null_handles_are_refused():
    L = rdcn.load()
    s, t, u = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    A = rdcn.RDCN_ERR_ARG
    assert L.rdcn_softmax_loss_workspace(None, 1, 8, 8, ctypes.byref(s), ctypes.byref(t), ctypes.byref(u)) == A
    assert L.rdcn_softmax_loss_forward(None, 1, 8, 8, None, None, None, None, 1.0, None, None, None, 0, None) == A
    assert L.rdcn_softmax_loss_grad(None, 1, 8, 8, None, None, None, None, 1.0, None, 1.0, None, None, None, None, None, 0,
                                    None) == A
    c = rdcn.RdcnAdamwConfig(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, None, None, None, 0, 0)
    lst = (rdcn.RdcnAdamwTensor * 1)()
    assert L.rdcn_adamw_step(None, ctypes.byref(c), lst, 1, None) == A
    assert L.rdcn_adamw_values(None, 1, None, None, 0, None, None) == A
    assert L.rdcn_grad_norm_workspace(None, lst, 1, ctypes.byref(s)) == A
    assert L.rdcn_grad_norm(None, lst, 1, 1.0, 1.0, None, None, 0, None) == A


def test_descriptors_check_their_tensors():
    def t(**kw):
        d = {k: torch.zeros(600) for k in ("param", "grad", "m", "v")}
        d.update(kw)
        return d

    lst = rdcn.adamw_tensors([t(), t(weight_decay=0.5, m=torch.zeros(600, dtype=torch.uint8), v=torch.zeros(600, dtype=torch.uint8),
                                     exps=torch.zeros(6, dtype=torch.uint8))])
    assert [x.n for x in lst] == [600, 600] and lst[1].weight_decay == 0.5 and [x.moments for x in lst] == [0, 1]
    for bad in (t(grad=torch.zeros(599)), t(m=torch.zeros(600, dtype=torch.uint8)), t(v=torch.zeros(601)),
                t(param=torch.zeros(1200)[::2]), t(master=torch.zeros(1)),
                t(m=torch.zeros(600, dtype=torch.uint8), v=torch.zeros(600, dtype=torch.uint8),
                  exps=torch.zeros(5, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            rdcn.adamw_tensors([bad])
