"""Python binding of the entry points of include/vmoe_train.h (ctypes).

Block norm, load-balance loss and AdamW of a sparse block's training step.
Functions have the names and argument order of the C calls and take torch
device tensors (or None for optional pointers); all arithmetic runs in
libvmoe.so. Beyond marshalling, the binding checks what a pointer cannot say:
a tensor's type, that it is contiguous, on the GPU and large enough
(ValueError); everything else is the library's status (VmoeError).
"""
from __future__ import annotations

import ctypes
import dataclasses
import math
import os

import torch

from . import vmoe as V
from .vmoe import VMOE_BF16, VMOE_F32, VmoeError, _check, _lib, _ptr, _stream  # noqa: F401

HEADER = os.path.join(os.path.dirname(V.HEADER), "vmoe_train.h")

VMOE_NORM_NONE, VMOE_NORM_RMS, VMOE_NORM_LAYER = range(3)
VMOE_STATE_F32, VMOE_STATE_8BIT = range(2)
VMOE_ADAMW_CHUNK = 8192
VMOE_ADAMW_PLAN_ENTRY_BYTES = 80
STATE_BLOCK = 128  # elements of an 8-bit state that share a scale byte

_TORCH = {VMOE_F32: torch.float32, VMOE_BF16: torch.bfloat16}
_DTYPE = {t: c for c, t in _TORCH.items()}


class NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_tokens", "n_groups", "d_model", "dtype", "stream_dtype", "dh_dtype", "pre_norm",
        "post_norm")] + [(n, ctypes.c_float) for n in (
            "eps", "residual_scale", "branch_scale")] + [("reserved", ctypes.c_int32)]


class _TensorStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "param", "master", "grad", "m", "v", "m_scale", "v_scale")] + [
        ("n", ctypes.c_int64), ("index0", ctypes.c_uint64), ("lr_mult", ctypes.c_double),
        ("weight_decay", ctypes.c_double)] + [(n, ctypes.c_int32) for n in (
            "param_dtype", "grad_dtype", "state", "reserved")]


class _Hyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [
        ("step", ctypes.c_int64), ("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


def _declare():
    P, Z, F = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    D, I32, I64 = ctypes.c_double, ctypes.c_int32, ctypes.c_int64
    N, T = ctypes.POINTER(NormShape), ctypes.POINTER(_TensorStruct)
    S = ctypes.POINTER(V.Shape)
    for name, res, args in (
            ("vmoe_block_norm_fwd", I32, [N] + [P] * 13),
            ("vmoe_block_norm_bwd_workspace_bytes", Z, [N]),
            ("vmoe_block_norm_bwd", I32, [N] + [P] * 19 + [Z, P]),
            ("vmoe_load_balance_loss_workspace_bytes", Z, [S]),
            ("vmoe_load_balance_loss", I32, [S] + [P] * 6 + [F, F] + [P] * 5 + [Z, P]),
            ("vmoe_adamw_plan_chunks", I64, [T, I32]),
            ("vmoe_adamw_plan", I32, [T, I32, P, Z]),
            ("vmoe_grad_norm_workspace_bytes", Z, [I64]),
            ("vmoe_grad_norm", I32, [P, I64, D, D, P, P, Z, P]),
            ("vmoe_adamw", I32, [P, I64, ctypes.POINTER(_Hyper), P, P]),
            ("vmoe_adamw_state_values", I32, [P, P, I32, I64, P, I32, P])):
        f = getattr(_lib, name)
        f.restype, f.argtypes = res, args


_declare()


def _tensor(name, t, dtype, numel):
    """Pointer of a contiguous device tensor of `dtype` with at least `numel`
    elements (None stays NULL)."""
    if t is None:
        return None
    if not (t.dtype == dtype and t.is_cuda and t.is_contiguous() and t.numel() >= numel):
        raise ValueError(f"{name}: a contiguous {dtype} tensor of at least {numel} elements on "
                         f"the GPU is wanted, got {t.dtype} {tuple(t.shape)}, strides "
                         f"{t.stride()}, on {t.device}")
    return t.data_ptr()


def _workspace(t):
    if t is None:
        return None, 0
    return _ptr(t), t.numel() * t.element_size()


# ------------------------------------------------------------------ block norm

def make_norm_shape(n_tokens, d_model, dtype, *, n_groups=1, stream_dtype=None, dh_dtype=VMOE_F32,
                    pre_norm=VMOE_NORM_LAYER, post_norm=VMOE_NORM_NONE, eps=1e-6,
                    residual_scale=1.0, branch_scale=1.0) -> NormShape:
    """stream_dtype None: as dtype; dh_dtype: f32 as the sparse layer's dx."""
    return NormShape(n_tokens, n_groups, d_model, dtype,
                     dtype if stream_dtype is None else stream_dtype, dh_dtype, pre_norm,
                     post_norm, eps, residual_scale, branch_scale, 0)


def _norm_types(s):
    """Torch types of the activations, the stream and dh; unknown ones are left
    to the library's check."""
    act = _TORCH.get(s.dtype, torch.float32)
    return act, _TORCH.get(s.stream_dtype, torch.float32), _TORCH.get(s.dh_dtype, torch.float32)


def vmoe_block_norm_fwd(shape, x, y, post_weight, post_bias, gate, row_scale, pre_weight, pre_bias,
                        x_out, h, post_stats, pre_stats, stream=None):
    act, res, _ = _norm_types(shape)
    n, d = shape.n_tokens, shape.d_model
    f32 = torch.float32
    _check("vmoe_block_norm_fwd", _lib.vmoe_block_norm_fwd(
        ctypes.byref(shape), _tensor("x", x, res, n * d), _tensor("y", y, act, n * d),
        _tensor("post_weight", post_weight, act, d), _tensor("post_bias", post_bias, act, d),
        _tensor("gate", gate, act, shape.n_groups * d), _tensor("row_scale", row_scale, f32, n),
        _tensor("pre_weight", pre_weight, act, d), _tensor("pre_bias", pre_bias, act, d),
        _tensor("x_out", x_out, res, n * d), _tensor("h", h, act, n * d),
        _tensor("post_stats", post_stats, f32, 2 * n), _tensor("pre_stats", pre_stats, f32, 2 * n),
        _stream(stream)))


def vmoe_block_norm_bwd_workspace_bytes(shape: NormShape) -> int:
    return int(_lib.vmoe_block_norm_bwd_workspace_bytes(ctypes.byref(shape)))


def vmoe_block_norm_bwd(shape, dx_out, dh, x_out, y, post_weight, post_bias, gate, row_scale,
                        pre_weight, post_stats, pre_stats, dx, dy, dpost_weight, dpost_bias, dgate,
                        dpre_weight, dpre_bias, workspace, stream=None):
    act, res, grad = _norm_types(shape)
    n, d = shape.n_tokens, shape.d_model
    f32 = torch.float32
    ws, ws_bytes = _workspace(workspace)
    _check("vmoe_block_norm_bwd", _lib.vmoe_block_norm_bwd(
        ctypes.byref(shape), _tensor("dx_out", dx_out, res, n * d), _tensor("dh", dh, grad, n * d),
        _tensor("x_out", x_out, res, n * d), _tensor("y", y, act, n * d),
        _tensor("post_weight", post_weight, act, d), _tensor("post_bias", post_bias, act, d),
        _tensor("gate", gate, act, shape.n_groups * d), _tensor("row_scale", row_scale, f32, n),
        _tensor("pre_weight", pre_weight, act, d), _tensor("post_stats", post_stats, f32, 2 * n),
        _tensor("pre_stats", pre_stats, f32, 2 * n), _tensor("dx", dx, res, n * d),
        _tensor("dy", dy, act, n * d), _tensor("dpost_weight", dpost_weight, f32, d),
        _tensor("dpost_bias", dpost_bias, f32, d),
        _tensor("dgate", dgate, f32, shape.n_groups * d),
        _tensor("dpre_weight", dpre_weight, f32, d), _tensor("dpre_bias", dpre_bias, f32, d), ws,
        ws_bytes, _stream(stream)))


# ------------------------------------------------------------------ load-balance loss

def vmoe_load_balance_loss_workspace_bytes(shape: V.Shape) -> int:
    return int(_lib.vmoe_load_balance_loss_workspace_bytes(ctypes.byref(shape)))


def vmoe_load_balance_loss(shape, logits, logit_bias, noise, probs, expert_idx, token_mask,
                           w_balance, w_z, losses, demand, mean_probs, dlogits, workspace,
                           stream=None):
    n, E, G = shape.n_tokens, shape.n_experts, shape.n_groups
    f32, i32 = torch.float32, torch.int32
    ws, ws_bytes = _workspace(workspace)
    _check("vmoe_load_balance_loss", _lib.vmoe_load_balance_loss(
        ctypes.byref(shape), _tensor("logits", logits, f32, n * E),
        _tensor("logit_bias", logit_bias, f32, E), _tensor("noise", noise, f32, n * E),
        _tensor("probs", probs, f32, n * E), _tensor("expert_idx", expert_idx, i32, n * shape.k),
        _tensor("token_mask", token_mask, torch.uint8, n), float(w_balance), float(w_z),
        _tensor("losses", losses, f32, 2 * G), _tensor("demand", demand, i32, G * E),
        _tensor("mean_probs", mean_probs, f32, G * E), _tensor("dlogits", dlogits, f32, n * E), ws,
        ws_bytes, _stream(stream)))


# ------------------------------------------------------------------ AdamW

@dataclasses.dataclass
class AdamWTensor:
    """One tensor of an AdamW step: see vmoe_adamw_tensor. The state is in 8
    bits where m and v are u8 (with scales), else in f32."""
    param: torch.Tensor
    grad: torch.Tensor
    m: torch.Tensor
    v: torch.Tensor
    master: torch.Tensor | None = None
    m_scale: torch.Tensor | None = None
    v_scale: torch.Tensor | None = None
    lr_mult: float = 1.0
    weight_decay: float = 0.0
    index0: int | None = None  # None: after the tensors before it

    def struct(self, index0: int) -> _TensorStruct:
        n = self.param.numel()
        bits8 = self.m.dtype == torch.uint8
        state = torch.uint8 if bits8 else torch.float32
        scales = -(-n // STATE_BLOCK)
        types = {"param": self.param.dtype, "grad": self.grad.dtype}
        for what, t in types.items():
            if t not in _DTYPE:
                raise ValueError(f"{what}: float32 or bfloat16 is wanted, got {t}")
        sized = (("grad", self.grad, n), ("m", self.m, n), ("v", self.v, n),
                 ("master", self.master, n), ("m_scale", self.m_scale, scales),
                 ("v_scale", self.v_scale, scales))
        for what, t, count in sized:
            if t is not None and t.numel() != count:
                raise ValueError(f"{what}: {count} elements are wanted, got {t.numel()}")
        u8 = torch.uint8
        return _TensorStruct(
            _tensor("param", self.param, self.param.dtype, n),
            _tensor("master", self.master, torch.float32, n),
            _tensor("grad", self.grad, self.grad.dtype, n), _tensor("m", self.m, state, n),
            _tensor("v", self.v, state, n), _tensor("m_scale", self.m_scale, u8, scales),
            _tensor("v_scale", self.v_scale, u8, scales), n, index0, self.lr_mult,
            self.weight_decay, _DTYPE[self.param.dtype], _DTYPE[self.grad.dtype],
            VMOE_STATE_8BIT if bits8 else VMOE_STATE_F32, 0)


class AdamWPlan:
    """The chunks of a set of tensors, on the GPU. It keeps the tensors alive;
    make a new one when a tensor is replaced."""

    def __init__(self, tensors, device="cuda"):
        self.tensors = list(tensors)
        array = (_TensorStruct * max(len(self.tensors), 1))()
        at = 0
        for i, t in enumerate(self.tensors):
            index0 = at if t.index0 is None else t.index0
            array[i] = t.struct(index0)
            at = index0 + -(-t.param.numel() // STATE_BLOCK) * STATE_BLOCK
        self.n_chunks = int(_lib.vmoe_adamw_plan_chunks(array, len(self.tensors)))
        if self.n_chunks < 0:
            raise VmoeError("vmoe_adamw_plan_chunks", V.VMOE_ERR_INVALID_ARG)
        host = torch.zeros(max(self.n_chunks * VMOE_ADAMW_PLAN_ENTRY_BYTES, 16), dtype=torch.uint8)
        _check("vmoe_adamw_plan", _lib.vmoe_adamw_plan(array, len(self.tensors), host.data_ptr(),
                                                       host.numel()))
        self.table = host.to(device)


def vmoe_grad_norm_workspace_bytes(plan: AdamWPlan) -> int:
    return int(_lib.vmoe_grad_norm_workspace_bytes(plan.n_chunks))


def vmoe_grad_norm(plan, max_norm, clip, workspace, grad_scale=1.0, stream=None):
    """clip [2] f32 out: norm of all gradients, factor for vmoe_adamw."""
    ws, ws_bytes = _workspace(workspace)
    _check("vmoe_grad_norm", _lib.vmoe_grad_norm(
        _ptr(plan.table), plan.n_chunks, float(grad_scale), float(max_norm),
        _tensor("clip", clip, torch.float32, 2), ws, ws_bytes, _stream(stream)))


def vmoe_adamw(plan, lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, clip=None,
               grad_scale=1.0, stream=None):
    """One step of every tensor of the plan; clip: vmoe_grad_norm's output or None."""
    hyper = _Hyper(lr, beta1, beta2, eps, grad_scale, step, seed & 0xFFFFFFFF, 0)
    _check("vmoe_adamw", _lib.vmoe_adamw(
        _ptr(plan.table), plan.n_chunks, ctypes.byref(hyper),
        _tensor("clip", clip, torch.float32, 2), _stream(stream)))


def vmoe_adamw_state_values(codes, scale, is_signed, out, stream=None):
    """Values of an 8-bit state into `out` (f32 or bf16)."""
    n = codes.numel()
    if out.dtype not in _DTYPE:
        raise ValueError(f"out: float32 or bfloat16 is wanted, got {out.dtype}")
    _check("vmoe_adamw_state_values", _lib.vmoe_adamw_state_values(
        _tensor("codes", codes, torch.uint8, n),
        _tensor("scale", scale, torch.uint8, -(-n // STATE_BLOCK)), int(bool(is_signed)), n,
        _tensor("out", out, out.dtype, n), _DTYPE[out.dtype], _stream(stream)))


def adamw_state(param, bits=32, master=None):
    """Zero states for `param`: the m, v, m_scale, v_scale (and, for a bf16
    param, master) arguments of AdamWTensor."""
    n, dev = param.numel(), param.device
    r = {}
    if param.dtype == torch.bfloat16:
        r["master"] = param.detach().float().reshape(-1).clone() if master is None else master
    if bits == 32:
        r["m"], r["v"] = (torch.zeros(n, dtype=torch.float32, device=dev) for _ in range(2))
    elif bits == 8:
        r["m"], r["v"] = (torch.zeros(n, dtype=torch.uint8, device=dev) for _ in range(2))
        blocks = math.ceil(n / STATE_BLOCK)
        r["m_scale"], r["v_scale"] = (torch.zeros(blocks, dtype=torch.uint8, device=dev)
                                      for _ in range(2))
    else:
        raise ValueError(f"bits: 8 or 32 is wanted, got {bits}")
    return r
