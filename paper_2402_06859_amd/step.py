"""Device buffers for one synthetic batch and the sequence of librdcn calls that
make one training step of the path: gather -> forward -> backward -> embedding
backward, with a head's loss between them (DeviceHead, DeviceClasses) and the
weights' update after them (DeviceAdamW). Only allocation and call order live
here; all arithmetic is in the library's kernels.
"""
from __future__ import annotations

import contextlib
import math
from typing import Callable, Optional, Sequence

import torch

from .rdcn import BF16, I64, Rdcn, adamw_tensors, config_for, muon_tensors
from .synth import Workload

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _on(stream):
    """Torch's own operations on `stream` (None: the current one)."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


class DeviceBatch:
    def __init__(self, wl: Workload, inp: dict, device: str = "cuda", id_type: str = "i64",
                 batch_max: Optional[int] = None):
        self.wl = wl
        self.B = inp["batch"]
        dev = torch.device(device)
        dt = _DT[wl.dtype]
        self.lib = Rdcn(config_for(wl, batch_max or self.B, id_type))
        d = self.lib.d
        assert d == wl.d
        ids = inp["ids"]
        self.ids = (ids if id_type == "i64" else ids.to(torch.int32)).contiguous().to(dev)
        self.offsets = None if inp["offsets"] is None else inp["offsets"].contiguous().to(dev)
        self.nnz = int(ids.numel())
        self.q_tables = inp["q_tables"].contiguous().to(dev)
        self.r_tables = inp["r_tables"].contiguous().to(dev)
        self.dense = inp["dense"].contiguous().to(dev)
        self.w_down = [w.contiguous().to(dev) for w in inp["w_down"]]
        self.u = [w.contiguous().to(dev) for w in inp["u"]]
        self.bias = [w.contiguous().to(dev) for w in inp["bias"]]
        self.grad_out = inp["grad_out"].contiguous().to(dev) if "grad_out" in inp else None
        B = self.B
        self.x0 = torch.empty((B, d), dtype=dt, device=dev)
        self.x_out = torch.empty((B, d), dtype=dt, device=dev)
        saved_b, scratch_b = self.lib.workspace_bytes(B)
        self.saved = torch.empty(max(saved_b, 1), dtype=torch.uint8, device=dev)
        self.scratch = torch.empty(max(scratch_b, 1), dtype=torch.uint8, device=dev)
        self.grad_x0 = torch.empty((B, d), dtype=torch.float32, device=dev)
        self.g_w_down = [torch.empty(w.shape, dtype=torch.float32, device=dev) for w in self.w_down]
        self.g_u = [torch.empty(w.shape, dtype=torch.float32, device=dev) for w in self.u]
        self.g_bias = [torch.empty(w.shape, dtype=torch.float32, device=dev) for w in self.bias]
        self.grad_q = torch.zeros(self.q_tables.shape, dtype=torch.float32, device=dev)
        self.grad_r = torch.zeros(self.r_tables.shape, dtype=torch.float32, device=dev)
        eb = self.lib.embed_backward_workspace(B, self.nnz)
        self.emb_scratch = torch.empty(max(eb, 1), dtype=torch.uint8, device=dev)

    # individual calls
    def gather(self, stream=None):
        self.lib.qr_embed_gather(self.B, self.ids, self.offsets, self.q_tables, self.r_tables, self.dense, self.x0,
                                 stream)

    def forward(self, stream=None):
        self.lib.rdcn_forward(self.B, self.x0, self.w_down, self.u, self.bias, self.x_out, self.saved, self.scratch,
                              stream)

    def backward(self, grad_out: Optional[torch.Tensor] = None, stream=None):
        g = self.grad_out if grad_out is None else grad_out
        self.lib.rdcn_backward(self.B, self.x0, self.w_down, self.u, self.bias, self.saved, g, self.grad_x0,
                               self.g_w_down, self.g_u, self.g_bias, self.scratch, stream)

    def embed_backward(self, grad_x0: Optional[torch.Tensor] = None, stream=None):
        self.lib.qr_embed_backward(self.B, self.nnz, self.ids, self.offsets, self.q_tables, self.r_tables,
                                   self.grad_x0 if grad_x0 is None else grad_x0, self.grad_q, self.grad_r,
                                   self.emb_scratch, stream)

    def trained(self):
        """(weight, gradient) of everything that the path trains."""
        return (list(zip(self.w_down, self.g_w_down)) + list(zip(self.u, self.g_u)) + list(zip(self.bias, self.g_bias)) +
                [(self.q_tables, self.grad_q), (self.r_tables, self.grad_r)])

    def zero_table_grads(self, stream=None):
        with _on(stream):
            self.grad_q.zero_()
            self.grad_r.zero_()

    def step(self, stream=None):
        """One pass of the whole path (table gradients accumulate)."""
        self.gather(stream)
        self.forward(stream)
        self.backward(stream=stream)
        self.embed_backward(stream=stream)


class DeviceHead:
    """Device buffers of the head after the cross stack (gated MLP, logit, isotonic
    calibration, log loss) on the handle `lib`, and its call order."""

    def __init__(self, lib: Rdcn, head, hinp: dict, B: int, device: str = "cuda"):
        from .rdcn import make_head_config
        dev = torch.device(device)
        self.lib = lib
        self.head = head
        self.B = B
        lib.head_configure(make_head_config(head.widths, head.gated, head.buckets, head.lo, head.step))
        keys = ["W", "b"] + (["G", "c"] if head.gated else [])
        self.params = {k: [t.contiguous().to(dev) for t in hinp[k]] for k in keys}
        for k in ("w_out", "b_out", "cal_w", "cal_b"):
            self.params[k] = hinp[k].contiguous().to(dev)
        self.e = hinp["e"].contiguous().to(dev)
        self.labels = hinp["labels"].contiguous().to(dev)
        self.g_cal_in = hinp["g_cal"].contiguous().to(dev) if "g_cal" in hinp else None
        self.x = hinp["x"].contiguous().to(dev) if "x" in hinp else None
        saved_b, scratch_b = lib.head_workspace_bytes(B)
        self.saved = torch.empty(max(saved_b, 1), dtype=torch.uint8, device=dev)
        self.scratch = torch.empty(max(scratch_b, 1), dtype=torch.uint8, device=dev)
        self.y = torch.empty(B, dtype=torch.float32, device=dev)
        self.y_cal = torch.empty(B, dtype=torch.float32, device=dev)
        self.loss = torch.empty(B, dtype=torch.float32, device=dev)
        self.g_cal = torch.empty(B, dtype=torch.float32, device=dev)
        self.grad_x = torch.empty((B, lib.d), dtype=torch.bfloat16, device=dev)
        self.grad_e = torch.empty(self.e.shape, dtype=torch.float32, device=dev)
        self.grads = {k: [torch.empty(t.shape, dtype=torch.float32, device=dev) for t in self.params[k]]
                      for k in keys}
        for k in ("w_out", "b_out", "cal_w", "cal_b"):
            self.grads[k] = torch.empty(self.params[k].shape, dtype=torch.float32, device=dev)

    def forward(self, x: Optional[torch.Tensor] = None, stream=None):
        self.lib.head_forward(self.B, self.x if x is None else x, self.e, self.params, self.y, self.y_cal,
                              self.saved, stream)

    def logloss(self, stream=None):
        """Mean log loss over the batch: per-sample losses and dLoss/dy_cal = (sigmoid - label) / B."""
        self.lib.head_logloss(self.B, self.y_cal, self.labels, 1.0 / max(self.B, 1), self.loss, self.g_cal, stream)

    def backward(self, x: Optional[torch.Tensor] = None, g_cal: Optional[torch.Tensor] = None, stream=None):
        self.lib.head_backward(self.B, self.x if x is None else x, self.e, self.params, self.saved,
                               self.g_cal if g_cal is None else g_cal, self.grad_x, self.grad_e, self.grads,
                               self.scratch, stream)

    def tower_step(self, db: "DeviceBatch", stream=None):
        """One training step of a Feed-style tower: gather -> cross stack -> head ->
        log loss -> head backward -> cross-stack backward -> embedding backward."""
        db.gather(stream)
        db.forward(stream)
        self.forward(db.x_out, stream)
        self.logloss(stream)
        self.backward(db.x_out, stream=stream)
        db.backward(self.grad_x, stream)
        db.embed_backward(stream=stream)


class DeviceClasses:
    """Softmax loss over a large set of classes (items, tokens) on x [B, dim], normally x_L of the
    handle `lib`: class weights w [classes, dim] of its storage type, labels [B] of its id type (below 0: a row
    without one), their gradients and the call's scratch. What does not fit is a ValueError: the kernels go by pointers alone."""

    def __init__(self, lib: Rdcn, w: torch.Tensor, labels: torch.Tensor, offset: Optional[torch.Tensor] = None,
                 row_weight: Optional[torch.Tensor] = None, logit_scale: float = 1.0):
        self.lib, self.w, self.labels, self.offset, self.row_weight = lib, w, labels, offset, row_weight
        self.logit_scale = logit_scale
        self.B = labels.numel()
        self.classes, self.dim = w.shape
        self._fits("w", w, _DT["bf16" if lib.cfg.dtype == BF16 else "f32"], self.classes * self.dim)
        self._fits("labels", labels, torch.int64 if lib.cfg.id_type == I64 else torch.int32, self.B)
        for name, t, n in (("offset", offset, self.classes), ("row_weight", row_weight, self.B)):
            if t is not None:
                self._fits(name, t, torch.float32, n)
        dev = w.device
        self.loss = torch.empty(self.B, dtype=torch.float32, device=dev)
        self.lse = torch.empty(self.B, dtype=torch.float32, device=dev)
        self.grad_x = torch.empty((self.B, self.dim), dtype=w.dtype, device=dev)
        self.grad_w = torch.empty_like(w)
        self.scratch = torch.empty(max(lib.softmax_loss_workspace(self.B, self.dim, self.classes)[:2]),
                                   dtype=torch.uint8, device=dev)

    def _fits(self, name, t, dtype, n):
        if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != self.w.device:
            raise ValueError("DeviceClasses: %s must be %d contiguous values of %s on %s" % (name, n, dtype, self.w.device))

    def trained(self):
        return [(self.w, self.grad_w)]

    def forward(self, x: torch.Tensor, stream=None):
        """Loss and lse of every row, without gradients."""
        self._fits("x", x, self.w.dtype, self.B * self.dim)
        self.lib.softmax_loss_forward(self.B, self.dim, self.classes, x, self.w, self.offset, self.labels,
                                      self.logit_scale, self.loss, self.lse, self.scratch, stream)

    def loss_grad(self, x: torch.Tensor, scale: Optional[float] = None, stream=None):
        """Loss of every row and the gradients of scale (1 / B) times their (weighted) sum."""
        self._fits("x", x, self.w.dtype, self.B * self.dim)
        self.lib.softmax_loss_grad(self.B, self.dim, self.classes, x, self.w, self.offset, self.labels,
                                   self.logit_scale, self.row_weight, 1.0 / max(self.B, 1) if scale is None else scale,
                                   self.loss, self.lse, self.grad_x, self.grad_w, self.scratch, stream)

    def train_step(self, db: DeviceBatch, opt: Optional["DeviceAdamW"] = None, stream=None):
        """One training step: gather -> cross stack -> softmax loss and its gradient -> cross-stack backward ->
        embedding backward -> update."""
        db.zero_table_grads(stream)
        db.gather(stream)
        db.forward(stream)
        self.loss_grad(db.x_out, stream=stream)
        db.backward(self.grad_x, stream)
        db.embed_backward(stream=stream)
        if opt is not None:
            opt.update(stream)


class DeviceChoices:
    """Learning from recorded choices over a large set of classes, and answering from them, on x [B, dim], normally x_L of the handle
    `lib`: class weights w [classes, dim] of its storage type, the chosen class of each row (labels [B] of its id type; below 0: a row
    without one), offsets per class (-inf masks one). forward leaves logprob, entropy and lse [B] and, with top, the most
    probable classes (top_ids, top_logprob [B, top]); backward takes the loss's gradients in logprob and entropy to grad_x and
    grad_w. keep: whether forward keeps every class's exponential (2 bytes each, 4 in float models) and so saves backward a product.
    What does not fit is a ValueError."""

    def __init__(self, lib: Rdcn, w: torch.Tensor, labels: torch.Tensor, offset: Optional[torch.Tensor] = None,
                 logit_scale: float = 1.0, top: int = 0, keep: bool = True):
        self.lib, self.w, self.labels, self.offset, self.logit_scale, self.top = lib, w, labels, offset, logit_scale, top
        self.B = labels.numel()
        self.classes, self.dim = w.shape
        dev = w.device
        for name, t in (("labels", labels), ("offset", offset)):
            if t is not None and t.device != dev:
                raise ValueError("DeviceChoices: %s must be on %s" % (name, dev))
        f = dict(dtype=torch.float32, device=dev)
        self.logprob, self.entropy, self.lse = (torch.empty(self.B, **f) for _ in range(3))
        self.top_ids = torch.empty((self.B, top), dtype=labels.dtype, device=dev) if top else None
        self.top_logprob = torch.empty((self.B, top), **f) if top else None
        self.stats = torch.empty((self.B, 4), **f)
        self.grad_x = torch.empty((self.B, self.dim), dtype=w.dtype, device=dev)
        self.grad_w = torch.empty_like(w)
        forward, kept, grad, _ = lib.logprobs_workspace(self.B, self.dim, self.classes, top)
        self.kept = torch.empty(max(kept, 256), dtype=torch.uint8, device=dev) if keep else None
        self.scratch = torch.empty(max(forward, grad, 256), dtype=torch.uint8, device=dev)

    def trained(self):
        return [(self.w, self.grad_w)]

    def forward(self, x: torch.Tensor, stream=None):
        self.lib.logprobs_forward(self.B, self.dim, self.classes, x, self.w, self.offset, self.labels, self.logit_scale,
                                  self.logprob, self.entropy, self.lse, self.scratch, top=self.top, top_ids=self.top_ids,
                                  top_logprob=self.top_logprob, stats=self.stats, kept=self.kept, stream=stream)

    def backward(self, x: torch.Tensor, grad_logprob: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor] = None,
                 stream=None):
        """The gradients of the loss of the last forward on the same x."""
        self.lib.logprobs_grad(self.B, self.dim, self.classes, x, self.w, self.offset, self.labels, self.logit_scale,
                               self.stats, grad_logprob, grad_entropy, self.grad_x, self.grad_w, self.scratch,
                               kept=self.kept, stream=stream)

    def train_step(self, db: DeviceBatch, upstream: Callable, opts: Sequence = (), stream=None):
        """One training step: gather -> cross stack -> log probabilities -> upstream(logprob, entropy), which returns the loss's
        gradients in them -> their gradient -> cross-stack backward -> embedding backward -> the updates of opts."""
        db.zero_table_grads(stream)
        db.gather(stream)
        db.forward(stream)
        self.forward(db.x_out, stream)
        with _on(stream):
            g, h = upstream(self.logprob, self.entropy)
        self.backward(db.x_out, g, h, stream)
        db.backward(self.grad_x, stream)
        db.embed_backward(stream=stream)
        for opt in opts:
            opt.update(stream)


class DeviceAdamW:
    """AdamW over (weight, gradient) pairs, or (weight, gradient, weight_decay) where a weight has a decay of its own (an
    embedding table often none); the others decay by weight_decay if they have more than one dimension. Moments in float
    or 8 bits, float masters of bf16 weights or none, and the gradients clipped to max_norm together. Rate and step number stand on the device, so that an update
    can be captured in a graph: change lr with set_lr. With max_norm, an update whose gradients' norm is not finite
    is left out whole: weights, moments and the step number stay."""

    def __init__(self, lib: Rdcn, pairs: Sequence, lr: float, weight_decay: float = 0.0, moments: str = "f32",
                 master: bool = True, max_norm: Optional[float] = None, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, seed: int = 0):
        self.lib, self.max_norm = lib, max_norm
        self.hyper = dict(beta1=beta1, beta2=beta2, eps=eps, stochastic=True, carry=True, seed=seed)
        self.tensors = []
        for p, g, *own in pairs:
            n, dev = p.numel(), p.device
            mt = torch.uint8 if moments == "8bit" else torch.float32
            t = {"param": p, "grad": g, "m": torch.zeros(n, dtype=mt, device=dev),
                 "v": torch.zeros(n, dtype=mt, device=dev), "weight_decay": own[0] if own else weight_decay if p.dim() > 1 else 0.0}
            if moments == "8bit":
                t["exps"] = torch.zeros(2 * -(-n // 256), dtype=torch.uint8, device=dev)
            if master and p.dtype == torch.bfloat16:
                t["master"] = p.float()
            self.tensors.append(t)
        self.list = adamw_tensors(self.tensors)
        dev = self.tensors[0]["param"].device
        self.lr = torch.full((1,), lr, dtype=torch.float32, device=dev)
        self.steps = torch.zeros(1, dtype=torch.int64, device=dev)
        self.norm = torch.zeros(2, dtype=torch.float32, device=dev)   # norm of the gradients, clip factor
        self.taken = torch.zeros(1, dtype=torch.bool, device=dev)     # whether the update is taken
        self.scratch = torch.empty(max(256, lib.grad_norm_workspace(self.list)), dtype=torch.uint8, device=dev)

    def set_lr(self, lr: float, stream=None):
        with _on(stream):
            self.lr.fill_(lr)

    def update(self, stream=None):
        clip = None
        if self.max_norm is not None:
            self.lib.grad_norm(self.list, 1.0, self.max_norm, self.norm, self.scratch, stream)
            clip = self.norm[1:]
        with _on(stream):
            if clip is None:
                self.steps.add_(1)
            else:  # (the factor is NaN where the norm is not finite; a step that is not taken has no part in 1 - beta^t)
                self.steps.add_(torch.eq(clip, clip, out=self.taken))
        self.lib.adamw_step(self.list, lr=0.0, device_lr=self.lr, device_step=self.steps, clip=clip, stream=stream,
                            **self.hyper)


class DeviceMuon:
    """Muon over (weight, gradient) pairs of matrices, or (weight, gradient, weight_decay), beside a DeviceAdamW for everything
    else. A matrix that stacks several maps steps them apart where each one's rows are a pair of their own. Every update's elements are
    of size 0.2 lr, whatever the matrix's shape, like AdamW's. Float masters of bf16 weights or none, and the
    gradients clipped to max_norm together. Rate and step number stand on the device: change lr with set_lr. With max_norm,
    an update whose gradients' norm is not finite is left out whole."""

    def __init__(self, lib: Rdcn, pairs: Sequence, lr: float, weight_decay: float = 0.0, momentum: float = 0.95,
                 nesterov: bool = True, master: bool = True, max_norm: Optional[float] = None, steps: int = 5,
                 coefficients=(3.4445, -4.7750, 2.0315), seed: int = 0):
        self.lib, self.max_norm = lib, max_norm
        self.hyper = dict(momentum=momentum, nesterov=nesterov, steps=steps, coefficients=coefficients, stochastic=True,
                          seed=seed)
        self.tensors = []
        for p, g, *own in pairs:
            t = {"param": p, "grad": g, "m": torch.zeros(p.shape, dtype=torch.float32, device=p.device),
                 "weight_decay": own[0] if own else weight_decay, "scale": 0.2 * math.sqrt(max(p.shape))}
            if master and p.dtype == torch.bfloat16:
                t["master"] = p.float()
            self.tensors.append(t)
        self.list = muon_tensors(self.tensors)
        # (the norm reads the gradients alone)
        self.norm_list = adamw_tensors([{"param": t["grad"], "grad": t["grad"], "m": t["m"], "v": t["m"]} for t in self.tensors])
        dev = self.tensors[0]["param"].device
        self.lr = torch.full((1,), lr, dtype=torch.float32, device=dev)
        self.steps = torch.zeros(1, dtype=torch.int64, device=dev)
        self.norm = torch.zeros(2, dtype=torch.float32, device=dev)   # norm of the gradients, clip factor
        self.scratch = torch.empty(max(256, lib.muon_workspace(self.list), lib.grad_norm_workspace(self.norm_list)),
                                   dtype=torch.uint8, device=dev)

    def set_lr(self, lr: float, stream=None):
        with _on(stream):
            self.lr.fill_(lr)

    def update(self, stream=None):
        clip = None
        if self.max_norm is not None:
            self.lib.grad_norm(self.norm_list, 1.0, self.max_norm, self.norm, self.scratch, stream)
            clip = self.norm[1:]
        with _on(stream):
            self.steps.add_(1)
        self.lib.muon_step(self.list, self.scratch, lr=0.0, device_lr=self.lr, device_step=self.steps, clip=clip,
                           stream=stream, **self.hyper)
