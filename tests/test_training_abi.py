"""The training calls (softmax loss, AdamW, gradient norm): struct layouts, and refusals that need no GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2402_06859_amd import rdcn
from paper_2402_06859_amd.step import DeviceAdamW, DeviceClasses

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


def test_descriptors_refuse_types_that_the_kernels_do_not_read():
    """The kernels go by the descriptor's types: a tensor of 2 bytes an element taken for one of 4 would be read and
    written past its end."""
    n = 600
    f, h, b, u8 = torch.float32, torch.float16, torch.bfloat16, torch.uint8

    def t(eight=False, **types):
        d = {k: torch.zeros(n, dtype=types.pop(k, f)) for k in ("param", "grad")}
        d.update({k: torch.zeros(n, dtype=types.pop(k, u8 if eight else f)) for k in ("m", "v")})
        if eight:
            d["exps"] = torch.zeros(6, dtype=types.pop("exps", u8))
        d.update({k: torch.zeros(n, dtype=v) for k, v in types.items()})
        return d

    fine = [t(), t(param=b), t(grad=b), t(param=b, master=f), t(eight=True), t(eight=True, param=b, grad=b, master=f)]
    lst = rdcn.adamw_tensors(fine)
    assert [(x.param_dtype, x.grad_dtype) for x in lst] == [(0, 0), (1, 0), (0, 1), (1, 0), (0, 0), (1, 1)]
    bad = [t(param=h), t(param=torch.float64), t(grad=h), t(grad=torch.float64), t(param=torch.int32), t(param=h, master=f),
           t(param=b, master=b), t(param=b, master=h), t(param=b, master=torch.float64), t(master=f), t(m=h, v=h),
           t(eight=True, exps=torch.int32), t(eight=True, exps=torch.int8),
           dict(t(eight=True), exps=torch.zeros(12, dtype=u8)[::2]), dict(t(eight=True), exps=None),
           dict(t(), grad=torch.zeros(n, device="meta")), dict(t(eight=True), exps=torch.zeros(6, dtype=u8, device="meta"))]
    no_exps = t(eight=True)
    del no_exps["exps"]
    for d in bad + [no_exps]:
        with pytest.raises(ValueError):
            rdcn.adamw_tensors([d])
    with pytest.raises(ValueError):
        rdcn.adamw_tensors([t(), {k: x.to("meta") for k, x in t().items()}])


class NoDevice:
    """The library's calls as far as DeviceClasses makes them, without a GPU."""

    def __init__(self, dtype, id_type):
        self.cfg = rdcn.make_config(8, 4, 16, 32, 8, 1, 25, 25, 600, dtype=dtype, id_type=id_type)
        self.calls = 0

    def softmax_loss_workspace(self, rows, dim, classes):
        return 256, 256, 256

    def softmax_loss_forward(self, *a):
        self.calls += 1

    softmax_loss_grad = softmax_loss_forward

    def grad_norm_workspace(self, tensors):
        return 256


@pytest.mark.parametrize("dtype,id_type", [("bf16", "i64"), ("bf16", "i32"), ("f32", "i64"), ("f32", "i32")])
def test_classes_refuse_tensors_that_the_kernels_would_read_past(dtype, id_type):
    B, dim, V = 6, 16, 10
    dt, other = (torch.bfloat16, torch.float32) if dtype == "bf16" else (torch.float32, torch.bfloat16)
    it, wrong = (torch.int64, torch.int32) if id_type == "i64" else (torch.int32, torch.int64)
    lib = NoDevice(dtype, id_type)
    w, y = torch.zeros(V, dim, dtype=dt), torch.zeros(B, dtype=it)
    dc = DeviceClasses(lib, w, y, offset=torch.zeros(V), row_weight=torch.ones(B))
    x = torch.zeros(B, dim, dtype=dt)
    dc.forward(x)
    dc.loss_grad(x)
    assert lib.calls == 2
    for bad in (x.to(other), x[:5], torch.zeros(B, dim + 8, dtype=dt), torch.zeros(B, 2 * dim, dtype=dt)[:, ::2],
                torch.zeros(B, 2 * dim, dtype=dt)[:, :dim], x.to("meta")):
        for call in (dc.forward, dc.loss_grad):
            with pytest.raises(ValueError):
                call(bad)
    for kw in (dict(w=w.to(other)), dict(w=w.half()), dict(w=torch.zeros(dim, V, dtype=dt).t()), dict(labels=y.to(wrong)),
               dict(labels=y.float()), dict(labels=torch.zeros(2 * B, dtype=it)[::2]), dict(offset=torch.zeros(V - 1)),
               dict(offset=torch.zeros(V, dtype=torch.bfloat16)), dict(row_weight=torch.ones(B, dtype=torch.float64)),
               dict(row_weight=torch.ones(B - 1)), dict(labels=y.to("meta"))):
        with pytest.raises(ValueError):
            DeviceClasses(**{**dict(lib=lib, w=w, labels=y), **kw})
    assert lib.calls == 2


def test_weights_with_a_decay_of_their_own():
    pair = lambda *shape: (torch.zeros(shape), torch.zeros(shape))
    opt = DeviceAdamW(NoDevice("f32", "i64"), [pair(4, 8), pair(8), (*pair(100, 4), 0.0), (*pair(8), 0.5), (*pair(4, 8), 0.25)],
                      lr=1e-3, weight_decay=0.125)
    assert [t.weight_decay for t in opt.list] == [0.125, 0.0, 0.0, 0.5, 0.25]


@pytest.mark.parametrize("name", ["_raw_stream", "_raw_device"])
def test_the_current_stream_without_torchs_private_calls(name, monkeypatch):
    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(rdcn, name, None)
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    assert rdcn._stream() == 77 and rdcn._stream(Stream()) == 77


def test_small_arguments_of_other_types_are_refused(monkeypatch):
    """What the kernels read as one float, one int64 or a byte per value and block."""
    lib = object.__new__(rdcn.Rdcn)  # a handle that refuses: nothing is launched
    lib.h = None
    lst = rdcn.adamw_tensors([{k: torch.zeros(300) for k in ("param", "grad", "m", "v")}])
    z = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype)
    u8, bf16 = torch.uint8, torch.bfloat16
    monkeypatch.setattr(rdcn, "_stream", lambda stream=None: None)
    for fine in (lambda: lib.grad_norm(lst, 1.0, 1.0, z(2), z(64)),
                 lambda: lib.adamw_step(lst, 1e-3, device_lr=z(1), device_step=z(1, torch.int64), clip=z(1)),
                 lambda: lib.adamw_values(z(300, u8), z(2, u8), True, z(300, bf16))):
        with pytest.raises(rdcn.RdcnError):  # the library's own refusal, of the handle
            fine()
    for bad in (lambda: lib.grad_norm(lst, 1.0, 1.0, z(1), z(64)), lambda: lib.grad_norm(lst, 1.0, 1.0, z(2, bf16), z(64)),
                lambda: lib.adamw_step(lst, 1e-3, device_lr=z(1, bf16)),
                lambda: lib.adamw_step(lst, 1e-3, device_step=z(1, torch.int32)),
                lambda: lib.adamw_step(lst, 1e-3, device_step=z(0, torch.int64)),
                lambda: lib.adamw_step(lst, 1e-3, clip=z(1, torch.float64)),
                lambda: lib.adamw_values(z(300, torch.int32), z(2, u8), True),
                lambda: lib.adamw_values(z(300, u8), z(1, u8), True), lambda: lib.adamw_values(z(600, u8)[::2], z(2, u8), True),
                lambda: lib.adamw_values(z(300, u8), z(2, u8), True, z(300)),
                lambda: lib.adamw_values(z(300, u8), z(2, u8), True, z(299, bf16))):
        with pytest.raises(ValueError):
            bad()
