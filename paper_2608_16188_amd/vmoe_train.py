"""Python binding of the entry points of include/vmoe_train.h.

Block norm, load-balance loss and AdamW of a sparse block's training step.
Functions have the names and argument order of the C calls and take torch
device tensors (or None for optional pointers); all arithmetic runs in
libvmoe.so. Marshalling runs in the extension module _train, which also checks
what a pointer cannot say: a tensor's type, that it is contiguous, on the
current GPU as the others are and large enough (ValueError); everything else is
the library's status (VmoeError). A missing library or extension raises at import.
"""
from __future__ import annotations

import ctypes
import dataclasses
import math
import os

import torch

from . import vmoe as V  # first: it loads libvmoe.so, which _train is linked to
from . import _train
from .vmoe import VMOE_BF16, VMOE_F32, VmoeError, _check, _lib  # noqa: F401

HEADER = os.path.join(os.path.dirname(V.HEADER), "vmoe_train.h")

VMOE_NORM_NONE, VMOE_NORM_RMS, VMOE_NORM_LAYER = range(3)
VMOE_STATE_F32, VMOE_STATE_8BIT = range(2)
STATE_BLOCK = 128  # elements of an 8-bit state that share a scale byte


class NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_tokens", "n_groups", "d_model", "dtype", "stream_dtype", "dh_dtype", "pre_norm",
        "post_norm")] + [(n, ctypes.c_float) for n in (
            "eps", "residual_scale", "branch_scale")] + [("reserved", ctypes.c_int32)]


def _declare():
    P, Z, I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
    for name, args in (("vmoe_block_norm_bwd_workspace_bytes", [P]),
                       ("vmoe_load_balance_loss_workspace_bytes", [P]),
                       ("vmoe_grad_norm_workspace_bytes", [I64])):
        f = getattr(_lib, name)
        f.restype, f.argtypes = Z, args


_declare()


# ------------------------------------------------------------------ block norm

def make_norm_shape(n_tokens, d_model, dtype, *, n_groups=1, stream_dtype=None, dh_dtype=VMOE_F32,
                    pre_norm=VMOE_NORM_LAYER, post_norm=VMOE_NORM_NONE, eps=1e-6,
                    residual_scale=1.0, branch_scale=1.0) -> NormShape:
    """stream_dtype None: as dtype; dh_dtype: f32 as the sparse layer's dx."""
    return NormShape(n_tokens, n_groups, d_model, dtype,
                     dtype if stream_dtype is None else stream_dtype, dh_dtype, pre_norm,
                     post_norm, eps, residual_scale, branch_scale, 0)


def vmoe_block_norm_fwd(shape, x, y, post_weight, post_bias, gate, row_scale, pre_weight, pre_bias,
                        x_out, h, post_stats, pre_stats, stream=None):
    _check("vmoe_block_norm_fwd", _train.block_norm_fwd(
        shape, x, y, post_weight, post_bias, gate, row_scale, pre_weight, pre_bias, x_out, h,
        post_stats, pre_stats, stream))


def vmoe_block_norm_bwd_workspace_bytes(shape: NormShape) -> int:
    return int(_lib.vmoe_block_norm_bwd_workspace_bytes(ctypes.byref(shape)))


def vmoe_block_norm_bwd(shape, dx_out, dh, x_out, y, post_weight, post_bias, gate, row_scale,
                        pre_weight, post_stats, pre_stats, dx, dy, dpost_weight, dpost_bias, dgate,
                        dpre_weight, dpre_bias, workspace, stream=None):
    _check("vmoe_block_norm_bwd", _train.block_norm_bwd(
        shape, dx_out, dh, x_out, y, post_weight, post_bias, gate, row_scale, pre_weight,
        post_stats, pre_stats, dx, dy, dpost_weight, dpost_bias, dgate, dpre_weight, dpre_bias,
        workspace, stream))


# ------------------------------------------------------------------ load-balance loss

def vmoe_load_balance_loss_workspace_bytes(shape: V.Shape) -> int:
    return int(_lib.vmoe_load_balance_loss_workspace_bytes(ctypes.byref(shape)))


def vmoe_load_balance_loss(shape, logits, logit_bias, noise, probs, expert_idx, token_mask,
                           w_balance, w_z, losses, demand, mean_probs, dlogits, workspace,
                           stream=None):
    _check("vmoe_load_balance_loss", _train.load_balance_loss(
        shape, logits, logit_bias, noise, probs, expert_idx, token_mask, w_balance, w_z, losses,
        demand, mean_probs, dlogits, workspace, stream))


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


class AdamWPlan:
    """The chunks of a set of tensors, on the GPU. It keeps the tensors alive;
    make a new one when a tensor is replaced or its rates change. The random
    numbers of 8-bit states start at the first tensor's index0 (0 where it gives
    none): two plans that take the same steps with one seed need an index0 of their
    own, or seeds of their own, to round with different ones."""

    def __init__(self, tensors, device="cuda"):
        self.tensors = list(tensors)
        status, self.n_chunks, table = _train.adamw_plan(self.tensors)
        _check("vmoe_adamw_plan", status)
        host = torch.frombuffer(bytearray(table), dtype=torch.uint8) if table else \
            torch.zeros(1, dtype=torch.uint8)
        self.table = host.to(device)
        if self.tensors and self.table.device != self.tensors[0].param.device:
            raise ValueError(f"device: the tensors are on {self.tensors[0].param.device}, the plan "
                             f"would be on {self.table.device}")
        self._entries = self.table if self.n_chunks else None


def vmoe_grad_norm_workspace_bytes(plan: AdamWPlan) -> int:
    return int(_lib.vmoe_grad_norm_workspace_bytes(plan.n_chunks))


def vmoe_grad_norm(plan, max_norm, clip, workspace, grad_scale=1.0, stream=None):
    """clip [2] f32 out: norm of all gradients, factor for vmoe_adamw."""
    _check("vmoe_grad_norm", _train.grad_norm(plan._entries, plan.n_chunks, grad_scale, max_norm,
                                              clip, workspace, stream))


def vmoe_adamw(plan, lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, clip=None,
               grad_scale=1.0, stream=None):
    """One step of every tensor of the plan; clip: vmoe_grad_norm's output or None.
    seed: 32 bits, of 8-bit states' random numbers. step, lr and seed are those of
    this call wherever it is captured and replayed."""
    _check("vmoe_adamw", _train.adamw(plan._entries, plan.n_chunks, lr, beta1, beta2, eps,
                                      grad_scale, step, seed, clip, stream))


def vmoe_adamw_state_values(codes, scale, is_signed, out, stream=None):
    """Values of an 8-bit state into `out` (f32 or bf16)."""
    _check("vmoe_adamw_state_values",
           _train.adamw_state_values(codes, scale, is_signed, out, stream))


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
