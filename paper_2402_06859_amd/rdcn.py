"""Python binding of librdcn (include/rdcn.h): argument marshalling only.

Every computation runs in the library's HIP kernels; torch is used for device
memory and the current stream. If the shared library is missing it is built
with hipcc; if it cannot be loaded, an error is raised (there is no fallback).
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librdcn.so")
MAX_LAYERS = 16

(RDCN_OK, RDCN_ERR_ARG, RDCN_ERR_SHAPE, RDCN_ERR_INDEX, RDCN_ERR_UNSUPPORTED, RDCN_ERR_WORKSPACE, RDCN_ERR_HIP,
 RDCN_ERR_RANGE) = range(8)
F32, BF16 = 0, 1
I32, I64 = 0, 1
COMBINE_MUL, COMBINE_SUM = 0, 1
MOMENTS_F32, MOMENTS_8BIT = 0, 1
ROUND_CARRY = 2   # with stochastic: RDCN_ROUND_CHANCE_CARRY
ACT_MODES = {"storage": 0, "hilo": 1, "f16": 2}   # rdcn_act_mode

EXPORTS = ["rdcn_create", "rdcn_destroy", "rdcn_dim", "rdcn_workspace_bytes", "qr_embed_gather",
           "qr_embed_backward_workspace", "qr_embed_backward", "rdcn_forward", "rdcn_backward",
           "rdcn_check_device_errors", "rdcn_status_string", "rdcn_profile_start", "rdcn_profile_stop",
           "qr_quantize_tables", "qr_embed_gather_q8", "rdcn_head_configure", "rdcn_head_workspace_bytes",
           "rdcn_head_forward", "rdcn_head_logloss", "rdcn_head_backward", "rdcn_set_side_stream",
           "qr_embed_backward_static", "rdcn_softmax_loss_workspace", "rdcn_softmax_loss_forward",
           "rdcn_softmax_loss_grad", "rdcn_adamw_step", "rdcn_adamw_values", "rdcn_grad_norm_workspace",
           "rdcn_grad_norm"]
EMBED_STATIC_SCRATCH_BYTES = 64 << 20

KERNELS = ["gather", "fwd_down_gemm", "fwd_attention", "fwd_up_gemm", "bwd_pointwise", "bwd_bias", "bwd_gu_gemm",
           "bwd_gh_gemm", "bwd_attention", "bwd_gw_gemm", "bwd_gx_gemm", "splitk_reduce", "emb_keys", "emb_sort",
           "emb_reduce", "gather_q8", "quantize", "head_gate", "head_fwd_gemm", "head_out", "head_loss",
           "head_out_bwd", "head_gw_gemm", "head_gx_gemm", "head_gate_bwd", "head_colsum", "emb_fused"]
MAX_HIDDEN = 8


class RdcnConfig(ctypes.Structure):
    _fields_ = [("batch_max", ctypes.c_int64), ("num_cat", ctypes.c_int32), ("emb_dim", ctypes.c_int32),
                ("num_dense", ctypes.c_int32), ("rank", ctypes.c_int32), ("num_layers", ctypes.c_int32),
                ("qr_rows_q", ctypes.c_int32), ("qr_rows_r", ctypes.c_int32), ("combine", ctypes.c_int32),
                ("multi_hot", ctypes.c_int32), ("id_type", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("activation_mode", ctypes.c_int32), ("vocab", ctypes.c_int64), ("attn_alpha", ctypes.c_float),
                ("skip_beta", ctypes.c_float), ("temperature", ctypes.c_float), ("parallel_branch", ctypes.c_int32),
                ("hashed", ctypes.c_int32), ("reserved2", ctypes.c_int32), ("hash_seed", ctypes.c_uint64)]


class RdcnWeights(ctypes.Structure):
    _fields_ = [("w_down", ctypes.c_void_p * MAX_LAYERS), ("u", ctypes.c_void_p * MAX_LAYERS),
                ("bias", ctypes.c_void_p * MAX_LAYERS)]


class RdcnHeadConfig(ctypes.Structure):
    _fields_ = [("num_hidden", ctypes.c_int32), ("hidden", ctypes.c_int32 * MAX_HIDDEN), ("gated", ctypes.c_int32),
                ("num_buckets", ctypes.c_int32), ("bucket_lo", ctypes.c_float), ("bucket_step", ctypes.c_float)]


class RdcnHeadWeights(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p * MAX_HIDDEN), ("b", ctypes.c_void_p * MAX_HIDDEN),
                ("gate_w", ctypes.c_void_p * MAX_HIDDEN), ("gate_b", ctypes.c_void_p * MAX_HIDDEN),
                ("w_out", ctypes.c_void_p), ("b_out", ctypes.c_void_p), ("cal_w", ctypes.c_void_p),
                ("cal_b", ctypes.c_void_p)]


class RdcnAdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("master", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("exps", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("weight_decay", ctypes.c_double), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("moments", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class RdcnAdamwConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("grad_scale", ctypes.c_double), ("step", ctypes.c_int64),
                ("device_lr", ctypes.c_void_p), ("device_step", ctypes.c_void_p), ("clip", ctypes.c_void_p),
                ("stochastic", ctypes.c_int32), ("seed", ctypes.c_uint32)]


def adamw_tensors(tensors: Sequence[dict]):
    """Descriptors of tensors to step, once for many steps. Each is a dict of device tensors
    param, grad, m, v and, where it has them, master and exps, and its weight_decay. The caller
    keeps the tensors alive. The kernels go by pointers alone, so what does not fit is a ValueError here."""
    out = (RdcnAdamwTensor * len(tensors))()
    for d, t in zip(out, tensors):
        n = t["param"].numel()
        for k in ("param", "master", "grad", "m", "v"):
            x = t.get(k)
            if x is not None and (x.numel() != n or not x.is_contiguous()):
                raise ValueError("adamw_tensors: %s must be contiguous, of as many elements as param" % k)
        for k in ("param", "grad"):
            if t[k].dtype not in (torch.float32, torch.bfloat16):
                raise ValueError("adamw_tensors: %s must be float32 or bfloat16, not %s" % (k, t[k].dtype))
        if t.get("master") is not None and (t["master"].dtype != torch.float32 or t["param"].dtype != torch.bfloat16):
            raise ValueError("adamw_tensors: a master is float32, of a bfloat16 param")
        if t["m"].dtype != t["v"].dtype or t["m"].dtype not in (torch.uint8, torch.float32):
            raise ValueError("adamw_tensors: m and v are both float32 or both uint8")
        if t["m"].dtype == torch.uint8:
            e = t.get("exps")
            if e is None or e.dtype != torch.uint8 or not e.is_contiguous() or e.numel() < 2 * -(-n // 256):
                raise ValueError("adamw_tensors: exps holds two exponents per 256 elements, contiguous uint8")
        if any(t[k].device != tensors[0]["param"].device for k in t if isinstance(t[k], torch.Tensor)):
            raise ValueError("adamw_tensors: tensors on more than one device")
        for k in ("param", "master", "grad", "m", "v", "exps"):
            x = t.get(k)
            setattr(d, k, None if x is None else x.data_ptr())
        d.n = t["param"].numel()
        d.weight_decay = t.get("weight_decay", 0.0)
        d.param_dtype = BF16 if t["param"].dtype == torch.bfloat16 else F32
        d.grad_dtype = BF16 if t["grad"].dtype == torch.bfloat16 else F32
        d.moments = MOMENTS_8BIT if t["m"].dtype == torch.uint8 else MOMENTS_F32
    return out


def make_head_config(hidden: Sequence[int], gated: bool, num_buckets: int, bucket_lo: float,
                     bucket_step: float) -> RdcnHeadConfig:
    c = RdcnHeadConfig()
    c.num_hidden = len(hidden)
    for i, n in enumerate(hidden):
        c.hidden[i] = n
    c.gated, c.num_buckets, c.bucket_lo, c.bucket_step = int(gated), num_buckets, bucket_lo, bucket_step
    return c


def head_weights(p: dict) -> RdcnHeadWeights:
    """p: W, b, (G, c), w_out, b_out, cal_w, cal_b (device tensors; G and c only when gated)."""
    w = RdcnHeadWeights()
    for l in range(len(p["W"])):
        w.w[l], w.b[l] = p["W"][l].data_ptr(), p["b"][l].data_ptr()
        if p.get("G") is not None:
            w.gate_w[l], w.gate_b[l] = p["G"][l].data_ptr(), p["c"][l].data_ptr()
    w.w_out, w.b_out = p["w_out"].data_ptr(), p["b_out"].data_ptr()
    w.cal_w, w.cal_b = p["cal_w"].data_ptr(), p["cal_b"].data_ptr()
    return w


class RdcnError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (fn, status_string(status), status))


_lib = None


def load(build_if_missing: bool = True):
    """Load librdcn.so (building it first if absent)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        if not build_if_missing:
            raise RuntimeError("librdcn.so is not built (%s)" % LIB_PATH)
        from . import build_lib
        build_lib.build()
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    st = ctypes.c_int
    L.rdcn_status_string.argtypes = [st]
    L.rdcn_status_string.restype = ctypes.c_char_p
    L.rdcn_create.argtypes = [ctypes.POINTER(RdcnConfig), ctypes.POINTER(vp)]
    L.rdcn_destroy.argtypes = [vp]
    L.rdcn_dim.argtypes = [vp, ctypes.POINTER(i64)]
    L.rdcn_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.qr_embed_gather.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp]
    L.qr_quantize_tables.argtypes = [vp, i64, vp, vp, vp, vp]
    L.qr_embed_gather_q8.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.qr_embed_backward_workspace.argtypes = [vp, i64, i64, ctypes.POINTER(sz)]
    L.qr_embed_backward.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.qr_embed_backward_static.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    L.rdcn_forward.argtypes = [vp, i64, vp, ctypes.POINTER(RdcnWeights), vp, vp, vp, vp]
    L.rdcn_backward.argtypes = [vp, i64, vp, ctypes.POINTER(RdcnWeights), vp, vp, vp, ctypes.POINTER(RdcnWeights),
                                vp, vp]
    L.rdcn_check_device_errors.argtypes = [vp, vp]
    L.rdcn_head_configure.argtypes = [vp, ctypes.POINTER(RdcnHeadConfig)]
    L.rdcn_head_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.rdcn_head_forward.argtypes = [vp, i64, vp, vp, ctypes.POINTER(RdcnHeadWeights), vp, vp, vp, vp]
    L.rdcn_head_logloss.argtypes = [vp, i64, vp, vp, ctypes.c_float, vp, vp, vp]
    L.rdcn_head_backward.argtypes = [vp, i64, vp, vp, ctypes.POINTER(RdcnHeadWeights), vp, vp, vp, vp,
                                     ctypes.POINTER(RdcnHeadWeights), vp, vp]
    f32 = ctypes.c_float
    L.rdcn_softmax_loss_workspace.argtypes = [vp, i64, i64, i64] + [ctypes.POINTER(sz)] * 3
    L.rdcn_softmax_loss_forward.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, f32, vp, vp, vp, sz, vp]
    L.rdcn_softmax_loss_grad.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, f32, vp, f32, vp, vp, vp, vp, vp, sz, vp]
    L.rdcn_adamw_step.argtypes = [vp, ctypes.POINTER(RdcnAdamwConfig), vp, ctypes.c_int32, vp]
    L.rdcn_adamw_values.argtypes = [vp, i64, vp, vp, ctypes.c_int32, vp, vp]
    L.rdcn_grad_norm_workspace.argtypes = [vp, vp, ctypes.c_int32, ctypes.POINTER(sz)]
    L.rdcn_grad_norm.argtypes = [vp, vp, ctypes.c_int32, f32, f32, vp, vp, sz, vp]
    L.rdcn_profile_start.argtypes = [vp, ctypes.c_int32, ctypes.c_uint32]
    L.rdcn_set_side_stream.argtypes = [vp, ctypes.c_int32]
    L.rdcn_profile_stop.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    for name in EXPORTS:
        if name != "rdcn_status_string":
            getattr(L, name).restype = st
    _lib = L
    return L


def status_string(s: int) -> str:
    return load().rdcn_status_string(s).decode()


def _check(fn: str, s: int):
    if s != RDCN_OK:
        raise RdcnError(fn, s)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _fits(fn: str, name: str, t: torch.Tensor, dtype: torch.dtype, n: int):
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError("%s: %s must be contiguous %s, %d or more" % (fn, name, dtype, n))


def _bytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.numel() * t.element_size()


# The raw handle of torch's current stream, which the object around it takes 2.7 us more to build: not part of torch's
# public interface, so a version without it takes the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None):
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def make_config(batch_max: int, num_cat: int, emb_dim: int, num_dense: int, rank: int, num_layers: int,
                qr_rows_q: int, qr_rows_r: int, vocab: int, combine: str = "sum", multi_hot: bool = False,
                id_type: str = "i64", dtype: str = "bf16", attn_alpha: float = 0.0, skip_beta: float = 1.0,
                temperature: float = 1.0, activation_mode: str = "storage",
                parallel_branch: bool = False, hashed: bool = False, hash_seed: int = 0) -> RdcnConfig:
    c = RdcnConfig()
    c.batch_max, c.num_cat, c.emb_dim, c.num_dense = batch_max, num_cat, emb_dim, num_dense
    c.rank, c.num_layers, c.qr_rows_q, c.qr_rows_r = rank, num_layers, qr_rows_q, qr_rows_r
    c.combine = COMBINE_MUL if combine == "mul" else COMBINE_SUM
    c.multi_hot = int(multi_hot)
    c.id_type = I64 if id_type == "i64" else I32
    c.dtype = BF16 if dtype == "bf16" else F32
    c.vocab = vocab
    c.attn_alpha, c.skip_beta, c.temperature = attn_alpha, skip_beta, temperature
    c.activation_mode = ACT_MODES[activation_mode]
    c.parallel_branch = int(parallel_branch)
    c.hashed = int(hashed)
    c.hash_seed = hash_seed
    return c


def config_for(wl, batch_max: Optional[int] = None, id_type: str = "i64") -> RdcnConfig:
    """Config of a synthetic workload (paper_2402_06859_amd.synth.Workload)."""
    return make_config(batch_max or wl.batch, wl.num_cat, wl.emb_dim, wl.num_dense, wl.rank, wl.num_layers,
                       wl.table_rows, wl.table_rows, 0 if wl.hashed else wl.vocab, wl.combine, wl.multi_hot, id_type,
                       wl.dtype, wl.alpha, wl.beta, wl.temperature, wl.act_mode, wl.parallel, wl.hashed,
                       wl.hash_seed)


def _weights(w_down: Sequence[torch.Tensor], u: Sequence[torch.Tensor], bias: Sequence[torch.Tensor]) -> RdcnWeights:
    w = RdcnWeights()
    for l, (a, b, c) in enumerate(zip(w_down, u, bias)):
        w.w_down[l], w.u[l], w.bias[l] = a.data_ptr(), b.data_ptr(), c.data_ptr()
    return w


class Rdcn:
    """One librdcn handle. Tensors are CUDA (HIP) tensors, contiguous, in the documented layouts."""

    def __init__(self, cfg: RdcnConfig):
        L = load()
        self.cfg = cfg
        h = ctypes.c_void_p()
        _check("rdcn_create", L.rdcn_create(ctypes.byref(cfg), ctypes.byref(h)))
        self.h = h
        d = ctypes.c_int64()
        _check("rdcn_dim", L.rdcn_dim(h, ctypes.byref(d)))
        self.d = d.value

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            load().rdcn_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- workspace
    def workspace_bytes(self, batch: int):
        s, t = ctypes.c_size_t(), ctypes.c_size_t()
        _check("rdcn_workspace_bytes", load().rdcn_workspace_bytes(self.h, batch, ctypes.byref(s), ctypes.byref(t)))
        return s.value, t.value

    def embed_backward_workspace(self, batch: int, nnz: int) -> int:
        s = ctypes.c_size_t()
        _check("qr_embed_backward_workspace", load().qr_embed_backward_workspace(self.h, batch, nnz, ctypes.byref(s)))
        return s.value

    # ---- entry points
    def qr_embed_gather(self, batch, ids, offsets, q_tables, r_tables, dense, x0, stream=None):
        _check("qr_embed_gather", load().qr_embed_gather(self.h, batch, _ptr(ids), _ptr(offsets), _ptr(q_tables),
                                                         _ptr(r_tables), _ptr(dense), _ptr(x0), _stream(stream)))

    def qr_quantize_tables(self, rows, tables, codes, params, stream=None):
        _check("qr_quantize_tables", load().qr_quantize_tables(self.h, rows, _ptr(tables), _ptr(codes), _ptr(params),
                                                               _stream(stream)))

    def qr_embed_gather_q8(self, batch, ids, offsets, q_codes, q_params, r_codes, r_params, dense, x0, stream=None):
        _check("qr_embed_gather_q8", load().qr_embed_gather_q8(
            self.h, batch, _ptr(ids), _ptr(offsets), _ptr(q_codes), _ptr(q_params), _ptr(r_codes), _ptr(r_params),
            _ptr(dense), _ptr(x0), _stream(stream)))

    def qr_embed_backward(self, batch, nnz, ids, offsets, q_tables, r_tables, grad_x0, grad_q, grad_r, scratch,
                          stream=None):
        _check("qr_embed_backward", load().qr_embed_backward(
            self.h, batch, nnz, _ptr(ids), _ptr(offsets), _ptr(q_tables), _ptr(r_tables), _ptr(grad_x0),
            _ptr(grad_q), _ptr(grad_r), _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))

    def qr_embed_backward_static(self, batch, nnz, ids, offsets, q_tables, r_tables, grad_x0, grad_q, grad_r,
                                 stream=None):
        _check("qr_embed_backward_static", load().qr_embed_backward_static(
            self.h, batch, nnz, _ptr(ids), _ptr(offsets), _ptr(q_tables), _ptr(r_tables), _ptr(grad_x0),
            _ptr(grad_q), _ptr(grad_r), _stream(stream)))

    def rdcn_forward(self, batch, x0, w_down, u, bias, x_out, saved, scratch=None, stream=None):
        w = _weights(w_down, u, bias)
        _check("rdcn_forward", load().rdcn_forward(self.h, batch, _ptr(x0), ctypes.byref(w), _ptr(x_out), _ptr(saved),
                                                   _ptr(scratch), _stream(stream)))

    def rdcn_backward(self, batch, x0, w_down, u, bias, saved, grad_out, grad_x0, g_w_down, g_u, g_bias, scratch,
                      stream=None):
        w = _weights(w_down, u, bias)
        g = _weights(g_w_down, g_u, g_bias)
        _check("rdcn_backward", load().rdcn_backward(self.h, batch, _ptr(x0), ctypes.byref(w), _ptr(saved),
                                                     _ptr(grad_out), _ptr(grad_x0), ctypes.byref(g), _ptr(scratch),
                                                     _stream(stream)))

    # ---- head (layers after the cross stack)
    def head_configure(self, cfg: RdcnHeadConfig):
        _check("rdcn_head_configure", load().rdcn_head_configure(self.h, ctypes.byref(cfg)))
        self.head_cfg = cfg

    def head_workspace_bytes(self, batch: int):
        s, t = ctypes.c_size_t(), ctypes.c_size_t()
        _check("rdcn_head_workspace_bytes",
               load().rdcn_head_workspace_bytes(self.h, batch, ctypes.byref(s), ctypes.byref(t)))
        return s.value, t.value

    def head_forward(self, batch, x, e_cal, params: dict, y_logit, y_cal, saved, stream=None):
        w = head_weights(params)
        _check("rdcn_head_forward", load().rdcn_head_forward(self.h, batch, _ptr(x), _ptr(e_cal), ctypes.byref(w),
                                                             _ptr(y_logit), _ptr(y_cal), _ptr(saved),
                                                             _stream(stream)))

    def head_logloss(self, batch, y_cal, labels, scale, loss=None, grad=None, stream=None):
        _check("rdcn_head_logloss", load().rdcn_head_logloss(self.h, batch, _ptr(y_cal), _ptr(labels), scale,
                                                             _ptr(loss), _ptr(grad), _stream(stream)))

    def head_backward(self, batch, x, e_cal, params: dict, saved, grad_ycal, grad_x, grad_e, grads: dict, scratch,
                      stream=None):
        w = head_weights(params)
        g = head_weights(grads)
        _check("rdcn_head_backward", load().rdcn_head_backward(
            self.h, batch, _ptr(x), _ptr(e_cal), ctypes.byref(w), _ptr(saved), _ptr(grad_ycal), _ptr(grad_x),
            _ptr(grad_e), ctypes.byref(g), _ptr(scratch), _stream(stream)))

    # ---- training over many classes
    def softmax_loss_workspace(self, rows: int, dim: int, classes: int):
        """Scratch bytes of (softmax_loss_forward, softmax_loss_grad), and the least that the gradient takes."""
        s, t, u = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        _check("rdcn_softmax_loss_workspace", load().rdcn_softmax_loss_workspace(
            self.h, rows, dim, classes, ctypes.byref(s), ctypes.byref(t), ctypes.byref(u)))
        return s.value, t.value, u.value

    def softmax_loss_forward(self, rows, dim, classes, x, w, offset, labels, logit_scale, loss, lse, scratch,
                             stream=None):
        _check("rdcn_softmax_loss_forward", load().rdcn_softmax_loss_forward(
            self.h, rows, dim, classes, _ptr(x), _ptr(w), _ptr(offset), _ptr(labels), logit_scale, _ptr(loss),
            _ptr(lse), _ptr(scratch), _bytes(scratch), _stream(stream)))

    def softmax_loss_grad(self, rows, dim, classes, x, w, offset, labels, logit_scale, row_weight, scale, loss, lse,
                          grad_x, grad_w, scratch, stream=None):
        _check("rdcn_softmax_loss_grad", load().rdcn_softmax_loss_grad(
            self.h, rows, dim, classes, _ptr(x), _ptr(w), _ptr(offset), _ptr(labels), logit_scale, _ptr(row_weight),
            scale, _ptr(loss), _ptr(lse), _ptr(grad_x), _ptr(grad_w), _ptr(scratch), _bytes(scratch),
            _stream(stream)))

    def grad_norm_workspace(self, tensors) -> int:
        s = ctypes.c_size_t()
        _check("rdcn_grad_norm_workspace", load().rdcn_grad_norm_workspace(self.h, tensors, len(tensors),
                                                                           ctypes.byref(s)))
        return s.value

    def grad_norm(self, tensors, grad_scale, max_norm, out, scratch, stream=None):
        """out (float [2]): the norm of all gradients of `tensors` (adamw_tensors) and the factor that clips it."""
        _fits("grad_norm", "out", out, torch.float32, 2)
        _check("rdcn_grad_norm", load().rdcn_grad_norm(self.h, tensors, len(tensors), grad_scale, max_norm, _ptr(out),
                                                       _ptr(scratch), _bytes(scratch), _stream(stream)))

    def adamw_step(self, tensors, lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1, grad_scale=1.0, clip=None,
                   stochastic=False, seed=0, device_lr=None, device_step=None, stream=None, carry=False):
        """One step over `tensors` (adamw_tensors). On the device: device_lr (float) and device_step (int64) in place of lr and
        step, and clip (float), the factor that grad_norm leaves. carry, with stochastic: the rounding to train 8-bit moments with."""
        if clip is not None:
            _fits("adamw_step", "clip", clip, torch.float32, 1)
        if device_lr is not None:
            _fits("adamw_step", "device_lr", device_lr, torch.float32, 1)
        if device_step is not None:
            _fits("adamw_step", "device_step", device_step, torch.int64, 1)
        c = RdcnAdamwConfig(lr, beta1, beta2, eps, grad_scale, step, _ptr(device_lr), _ptr(device_step), _ptr(clip),
                            int(stochastic) | (ROUND_CARRY if carry else 0), seed & 0xFFFFFFFF)
        _check("rdcn_adamw_step", load().rdcn_adamw_step(self.h, ctypes.byref(c), tensors, len(tensors),
                                                         _stream(stream)))

    def adamw_values(self, codes, exps, signed: bool, out=None, stream=None):
        """The values (bf16) that 8-bit moments stand for."""
        n = codes.numel()
        if (codes.dtype is not torch.uint8 or exps.dtype is not torch.uint8 or exps.numel() * 256 < n or
                not codes.is_contiguous() or not exps.is_contiguous()):
            raise ValueError("adamw_values: codes and one exponent for 256 of them, both contiguous uint8")
        if out is None:
            out = torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device)
        else:
            _fits("adamw_values", "out", out, torch.bfloat16, n)
        _check("rdcn_adamw_values", load().rdcn_adamw_values(self.h, n, _ptr(codes), _ptr(exps), int(signed),
                                                             _ptr(out), _stream(stream)))
        return out

    def profile_start(self, max_launches: int = 8192, kernels=None):
        """Time the launches of `kernels` (names from KERNELS; all when None)."""
        mask = 0xFFFFFFFF if kernels is None else sum(1 << KERNELS.index(k) for k in kernels)
        _check("rdcn_profile_start", load().rdcn_profile_start(self.h, max_launches, mask))

    def profile_stop(self) -> dict:
        """{kernel: (total_ms, launches)} of the launches timed since profile_start."""
        n = len(KERNELS)
        ms = (ctypes.c_double * n)()
        cnt = (ctypes.c_int64 * n)()
        _check("rdcn_profile_stop", load().rdcn_profile_stop(self.h, ms, cnt))
        return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNELS)}

    def set_side_stream(self, enable: bool):
        """Run the backward's weight-gradient work on the handle's second stream (default) or not."""
        _check("rdcn_set_side_stream", load().rdcn_set_side_stream(self.h, int(enable)))

    def check_device_errors(self, stream=None) -> int:
        """Synchronise and return (and clear) the device error status (RDCN_OK, RDCN_ERR_INDEX or
        RDCN_ERR_RANGE)."""
        return load().rdcn_check_device_errors(self.h, _stream(stream))
