"""Shared pieces of the tests of vmoe_train.h: float64 references, bounds and
the C structures."""
import ctypes

import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

U = 2.0 ** -24    # half an ulp of f32, relative
UB = 2.0 ** -8    # of bf16
NORMS = {"none": T.VMOE_NORM_NONE, "rms": T.VMOE_NORM_RMS, "layer": T.VMOE_NORM_LAYER}
DTYPES = {"f32": V.VMOE_F32, "bf16": V.VMOE_BF16}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class TensorStruct(ctypes.Structure):
    """vmoe_adamw_tensor."""
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "param", "master", "grad", "m", "v", "m_scale", "v_scale")] + [
        ("n", ctypes.c_int64), ("index0", ctypes.c_uint64), ("lr_mult", ctypes.c_double),
        ("weight_decay", ctypes.c_double)] + [(n, ctypes.c_int32) for n in (
            "param_dtype", "grad_dtype", "state", "reserved")]


class Hyper(ctypes.Structure):
    """vmoe_adamw_hyper."""
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [
        ("step", ctypes.c_int64), ("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


def close(name, got, ref, bound):
    """|got - ref| <= bound element by element (NaN nowhere)."""
    got, ref, bound = got.detach().double().cpu(), ref.double().cpu(), bound.double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all(), f"{name}: not finite"
    over = (got - ref).abs() - bound
    at = int(over.reshape(-1).argmax())
    assert over.max() <= 0, (
        f"{name}[{at}]: got {got.reshape(-1)[at]:.9g}, wanted {ref.reshape(-1)[at]:.9g} "
        f"within {bound.expand_as(got).reshape(-1)[at]:.3g}")


def rounding(dtype, ref):
    """One rounding of values near `ref` to an output's type."""
    return (UB if dtype == "bf16" else U) * 1.01 * ref.abs()


def same_bits(a, b):
    a, b = a.detach().cpu().contiguous(), b.detach().cpu().contiguous()
    return a.shape == b.shape and a.dtype == b.dtype and \
        torch.equal(a.view(torch.uint8), b.view(torch.uint8))
