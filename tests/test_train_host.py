"""Host-side checks of vmoe_train.h's calls (no GPU, nothing is launched):
exported symbols, refusals before anything is enqueued, the AdamW plan's
contents, and the binding's own checks."""
import ctypes
import math
import re
import struct
import subprocess

import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

from .train_common import Hyper, TensorStruct

FAKE = 0x10000  # 16-byte aligned, never dereferenced
BAD, UNS, WS = V.VMOE_ERR_INVALID_ARG, V.VMOE_ERR_UNSUPPORTED, V.VMOE_ERR_WORKSPACE
P, Z, I32, I64, D = (ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64,
                     ctypes.c_double)
SIGNATURES = {
    "vmoe_block_norm_fwd": (I32, [P] * 14),
    "vmoe_block_norm_bwd": (I32, [P] * 20 + [Z, P]),
    "vmoe_load_balance_loss": (I32, [P] * 7 + [ctypes.c_float] * 2 + [P] * 5 + [Z, P]),
    "vmoe_adamw_plan_chunks": (I64, [P, I32]),
    "vmoe_adamw_plan": (I32, [P, I32, P, Z]),
    "vmoe_grad_norm": (I32, [P, I64, D, D, P, P, Z, P]),
    "vmoe_adamw": (I32, [P, I64, P, P, P]),
    "vmoe_adamw_state_values": (I32, [P, P, I32, I64, P, I32, P]),
}


def call(name, *args):
    f = ctypes.CDLL(V.LIB_PATH)[name]  # a function object of its own
    f.restype, f.argtypes = SIGNATURES[name]
    return f(*args)


def test_declared_symbols_are_exported():
    text = open(T.HEADER).read()
    declared = set(re.findall(r"^\s*[\w\s\*]+?\b(vmoe_\w+)\s*\(", text, re.M))
    assert len(declared) == 11, declared
    out = subprocess.check_output(["nm", "-D", "--defined-only", V.LIB_PATH], text=True)
    exported = {line.split()[-1] for line in out.splitlines() if line.strip()}
    assert declared <= exported, declared - exported
    for s in declared:
        assert hasattr(T, s) or s in ("vmoe_adamw_plan", "vmoe_adamw_plan_chunks"), s


def _norm(**kw):
    base = dict(n_tokens=8, d_model=64, dtype=V.VMOE_BF16)
    base.update(kw)
    return T.make_norm_shape(base.pop("n_tokens"), base.pop("d_model"), base.pop("dtype"), **base)


@pytest.mark.parametrize("kw, status", [
    (dict(d_model=12), BAD), (dict(d_model=0), BAD), (dict(n_tokens=-1), BAD),
    (dict(n_tokens=9, n_groups=2), BAD), (dict(n_groups=0), BAD), (dict(dtype=2), BAD),
    (dict(stream_dtype=7), BAD), (dict(dh_dtype=-1), BAD), (dict(pre_norm=3), BAD),
    (dict(post_norm=-1), BAD), (dict(eps=0.0), BAD), (dict(eps=math.nan), BAD),
    (dict(eps=math.inf), BAD), (dict(residual_scale=math.inf), BAD),
    (dict(branch_scale=math.nan), BAD), (dict(dtype=V.VMOE_F32, stream_dtype=V.VMOE_BF16), BAD),
    (dict(dtype=V.VMOE_F32, dh_dtype=V.VMOE_BF16), BAD), (dict(d_model=16392), UNS),
    (dict(n_tokens=(1 << 30) + 1), UNS),
])
def test_norm_shapes_refused(kw, status):
    s = _norm(**kw)
    b = ctypes.byref(s)
    assert T.vmoe_block_norm_bwd_workspace_bytes(s) == 0
    assert call("vmoe_block_norm_fwd", b, *([FAKE] * 2), None, None, None, None, *([FAKE] * 4),
                None, FAKE, None) == status
    assert call("vmoe_block_norm_bwd", b, *([FAKE] * 4), *([None] * 4), FAKE, None, *([FAKE] * 3),
                None, None, None, FAKE, FAKE, FAKE, 1 << 40, None) == status
    s.reserved = 1
    assert call("vmoe_block_norm_fwd", b, *([FAKE] * 13)) == BAD


def _fwd(s, **kw):
    """x, y, post_w, post_b, gate, row_scale, pre_w, pre_b, x_out, h, post_stats, pre_stats"""
    a = dict(x=FAKE, y=FAKE, post_w=None, post_b=None, gate=FAKE, row=FAKE, pre_w=FAKE, pre_b=FAKE,
             x_out=FAKE, h=FAKE, post_stats=None, pre_stats=FAKE)
    a.update(kw)
    return call("vmoe_block_norm_fwd", ctypes.byref(s), *a.values(), None)


def test_norm_forward_pointers_refused():
    s = _norm()
    for kw in (dict(x=None), dict(x=FAKE + 8), dict(x_out=None), dict(h=None),
               dict(pre_stats=None), dict(gate=FAKE + 2), dict(row=FAKE + 4), dict(y=FAKE + 1),
               dict(post_w=FAKE), dict(post_b=FAKE),           # no post norm
               dict(y=None)):                                  # gate and row scale without a block
        assert _fwd(s, **kw) == BAD, kw
    post = _norm(post_norm=T.VMOE_NORM_RMS)
    assert _fwd(post) == BAD                                   # post_stats missing
    assert _fwd(post, post_stats=FAKE, y=None, gate=None, row=None) == BAD
    none = _norm(pre_norm=T.VMOE_NORM_NONE)
    assert _fwd(none) == BAD                                   # weights of a norm that is not there
    assert _fwd(none, y=None, gate=None, row=None, pre_w=None, pre_b=None) == BAD  # nothing to do
    assert call("vmoe_block_norm_fwd", None, *([FAKE] * 13)) == BAD


def _bwd(s, ws=1 << 30, workspace=FAKE, **kw):
    a = dict(dx_out=FAKE, dh=FAKE, x_out=FAKE, y=FAKE, post_w=None, post_b=None, gate=FAKE,
             row=FAKE, pre_w=FAKE, post_stats=None, pre_stats=FAKE, dx=FAKE, dy=FAKE, dpost_w=None,
             dpost_b=None, dgate=FAKE, dpre_w=FAKE, dpre_b=FAKE)
    a.update(kw)
    return call("vmoe_block_norm_bwd", ctypes.byref(s), *a.values(), workspace, ws, None)


def test_norm_backward_pointers_refused():
    s = _norm()
    for kw in (dict(dh=None), dict(x_out=None), dict(pre_stats=None), dict(dx=None), dict(dy=None),
               dict(dgate=FAKE + 8), dict(dpost_w=FAKE), dict(dpost_b=FAKE), dict(y=None),
               dict(dx_out=FAKE + 4)):
        assert _bwd(s, **kw) == BAD, kw
    assert _bwd(s, ws=8) == WS
    assert _bwd(s, workspace=None) == WS
    assert _bwd(s, workspace=FAKE + 4) == WS
    none = _norm(pre_norm=T.VMOE_NORM_NONE)
    assert _bwd(none, pre_w=None, dpre_w=None, dpre_b=None) == BAD   # dh without a norm
    assert _bwd(none, dh=None, pre_w=None, dpre_b=None) == BAD       # dpre_w without a norm


def test_load_balance_refused():
    s = V.make_shape(64, 2, 64, 64, 8, 2, 1.0, V.VMOE_F32)
    ok = [FAKE, FAKE, FAKE, FAKE, FAKE, FAKE]
    out = [FAKE, FAKE, FAKE, FAKE]
    b = ctypes.byref(s)

    def go(i=None, o=None, w=(0.1, 0.1), ws=1 << 30, p=FAKE, value=None):
        a, r = list(ok), list(out)
        if i is not None:
            a[i] = value
        if o is not None:
            r[o] = value
        return call("vmoe_load_balance_loss", b, *a, *w, *r, p, ws, None)

    for i in (0, 3, 4):
        assert go(i=i) == BAD
    for i in range(6):
        assert go(i=i, value=FAKE + 4) == BAD
    for o in (0, 1, 3):
        assert go(o=o) == BAD
    assert go(o=2, value=FAKE + 8) == BAD
    assert go(w=(math.nan, 0.0)) == BAD and go(w=(0.0, math.inf)) == BAD
    assert go(ws=T.vmoe_load_balance_loss_workspace_bytes(s) - 1) == WS
    assert go(p=None) == WS
    s.k = 9
    assert go() == BAD and T.vmoe_load_balance_loss_workspace_bytes(s) == 0


def _tensor(**kw):
    t = TensorStruct(FAKE, None, FAKE, FAKE, FAKE, None, None, 100, 0, 1.0, 0.0, V.VMOE_F32,
                     V.VMOE_F32, T.VMOE_STATE_F32, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


BF16 = dict(param_dtype=V.VMOE_BF16, master=FAKE)
BITS8 = dict(state=T.VMOE_STATE_8BIT, m_scale=FAKE, v_scale=FAKE)


@pytest.mark.parametrize("kw", [
    dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=FAKE + 4),
    dict(grad=FAKE + 8), dict(m=FAKE + 4), dict(v=FAKE + 8), dict(n=-1), dict(param_dtype=2),
    dict(grad_dtype=-1), dict(state=2), dict(reserved=1), dict(master=FAKE),
    dict(param_dtype=V.VMOE_BF16), dict(m_scale=FAKE), dict(v_scale=FAKE),
    dict(state=T.VMOE_STATE_8BIT), dict(BITS8, m_scale=None), dict(BITS8, v_scale=None),
    dict(BITS8, m=FAKE + 2), dict(index0=64), dict(lr_mult=-1.0), dict(lr_mult=math.inf),
    dict(weight_decay=math.nan), dict(weight_decay=-0.1), dict(BF16, master=FAKE + 4),
])
def test_adamw_tensors_refused(kw):
    t = (TensorStruct * 2)(_tensor(), _tensor(**kw))
    host = (ctypes.c_uint64 * 100)()
    assert call("vmoe_adamw_plan_chunks", t, 2) == -1
    assert call("vmoe_adamw_plan", t, 2, host, 800) == BAD


def test_adamw_plan_limits():
    host = (ctypes.c_uint64 * 100)()
    t = (TensorStruct * 1)(_tensor(n=3 * 8192 + 1))
    assert call("vmoe_adamw_plan_chunks", t, 1) == 4
    assert call("vmoe_adamw_plan", t, 1, host, 4 * 80 - 1) == WS
    assert call("vmoe_adamw_plan", t, 1, None, 1 << 20) == WS
    assert call("vmoe_adamw_plan", t, 1, host, 4 * 80) == V.VMOE_OK
    assert call("vmoe_adamw_plan_chunks", None, 1) == -1
    assert call("vmoe_adamw_plan_chunks", t, -1) == -1
    assert call("vmoe_adamw_plan_chunks", None, 0) == 0
    huge = (TensorStruct * 1)(_tensor(n=1 << 62))
    assert call("vmoe_adamw_plan_chunks", huge, 1) == -1
    assert call("vmoe_adamw_plan", huge, 1, host, 800) == UNS
    empty = (TensorStruct * 1)(_tensor(n=0, param=None, grad=None, m=None, v=None))
    assert call("vmoe_adamw_plan_chunks", empty, 1) == 0


def test_adamw_plan_contents():
    """Addresses, counts and random-number indexes of every chunk."""
    n = 2 * 8192 + 77
    a = _tensor(n=n, param=0x100000, grad=0x200000, m=0x300000, v=0x400000, index0=1 << 33,
                lr_mult=0.5, weight_decay=0.25, grad_dtype=V.VMOE_BF16)
    b = _tensor(**BITS8, n=5)
    c = _tensor(**BF16, n=8192)
    t = (TensorStruct * 3)(a, b, c)
    host = (ctypes.c_uint8 * (5 * 80))()
    assert call("vmoe_adamw_plan_chunks", t, 3) == 5
    assert call("vmoe_adamw_plan", t, 3, host, len(host)) == V.VMOE_OK
    rows = [struct.unpack_from("<7QQiIff", bytes(host), 80 * i) for i in range(5)]
    for i in range(3):
        o = 8192 * i
        assert rows[i][:7] == (0x100000 + 4 * o, 0, 0x200000 + 2 * o, 0x300000 + 4 * o,
                               0x400000 + 4 * o, 0, 0)
        assert rows[i][7] == (1 << 33) + o and rows[i][8] == min(8192, n - o)
        assert rows[i][10:] == (0.5, 0.25)
    assert rows[3][8] == 5 and rows[4][8] == 8192
    assert len({rows[0][9], rows[3][9], rows[4][9]}) == 3


def _hyper(**kw):
    h = Hyper(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0, 0)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


@pytest.mark.parametrize("kw", [
    dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
    dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-40), dict(eps=math.inf), dict(step=0),
    dict(grad_scale=math.inf), dict(reserved=1),
])
def test_adamw_scalars_refused(kw):
    assert call("vmoe_adamw", FAKE, 1, ctypes.byref(_hyper(**kw)), None, None) == BAD


def test_adamw_calls_refused():
    h = ctypes.byref(_hyper())
    assert call("vmoe_adamw", None, 1, h, None, None) == BAD
    assert call("vmoe_adamw", FAKE, -1, h, None, None) == BAD
    assert call("vmoe_adamw", FAKE, 1 << 31, h, None, None) == BAD
    assert call("vmoe_adamw", FAKE, 1, None, None, None) == BAD
    assert call("vmoe_adamw", FAKE, 1, h, FAKE + 4, None) == BAD
    assert call("vmoe_adamw", None, 0, h, None, None) == V.VMOE_OK  # nothing to do
    norm = lambda *a: call("vmoe_grad_norm", *a, None)  # noqa: E731
    assert norm(None, 1, 1.0, 1.0, FAKE, FAKE, 1 << 20) == BAD
    assert norm(FAKE, 1, math.nan, 1.0, FAKE, FAKE, 1 << 20) == BAD
    assert norm(FAKE, 1, 1.0, 0.0, FAKE, FAKE, 1 << 20) == BAD
    assert norm(FAKE, 1, 1.0, math.nan, FAKE, FAKE, 1 << 20) == BAD
    assert norm(FAKE, 1, 1.0, 1.0, None, FAKE, 1 << 20) == BAD
    assert norm(FAKE, 100, 1.0, 1.0, FAKE, FAKE, 8) == WS
    assert norm(FAKE, 1, 1.0, 1.0, FAKE, None, 1 << 20) == WS
    val = lambda *a: call("vmoe_adamw_state_values", *a, None)  # noqa: E731
    assert val(FAKE + 2, FAKE, 1, 5, FAKE, 0) == BAD
    assert val(FAKE, None, 1, 5, FAKE, 0) == BAD
    assert val(FAKE, FAKE, 2, 5, FAKE, 0) == BAD
    assert val(FAKE, FAKE, 1, -5, FAKE, 0) == BAD
    assert val(FAKE, FAKE, 1, 5, FAKE, 3) == BAD
    assert val(None, None, 0, 0, None, 1) == V.VMOE_OK


def test_binding_refuses_what_a_pointer_cannot_say():
    s = _norm()
    x = torch.zeros(8, 64, dtype=torch.bfloat16)
    rest = [None] * 11
    with pytest.raises(ValueError, match="x: .*not on the GPU"):
        T.vmoe_block_norm_fwd(s, x, *rest)
    with pytest.raises(ValueError, match="x: .*BFloat16.*got Float"):
        T.vmoe_block_norm_fwd(s, x.float(), *rest)
    with pytest.raises(ValueError, match="not contiguous"):
        T.vmoe_block_norm_fwd(s, torch.zeros(64, 8, dtype=torch.bfloat16).t(), *rest)
    with pytest.raises(TypeError, match="x: a tensor or None"):
        T.vmoe_block_norm_fwd(s, 5, *rest)
    with pytest.raises(TypeError):
        T.vmoe_block_norm_fwd(V.make_shape(8, 1, 64, 64, 8, 2, 1.0, 1), x, *rest)
    f = torch.zeros(4)
    with pytest.raises(ValueError, match="param"):
        T.AdamWPlan([T.AdamWTensor(f.double(), f, f, f)], device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        T.AdamWPlan([T.AdamWTensor(f, f, f, f)], device="cpu")
    assert T.AdamWPlan([], device="cpu").n_chunks == 0


def test_new_states():
    p = torch.zeros(3, 50, dtype=torch.bfloat16)
    s = T.adamw_state(p, bits=8)
    assert s["master"].shape == (150,) and s["m"].dtype == torch.uint8
    assert s["m_scale"].numel() == 2 and set(s) == {"master", "m", "v", "m_scale", "v_scale"}
    assert set(T.adamw_state(p.float())) == {"m", "v"}
    with pytest.raises(ValueError):
        T.adamw_state(p, bits=4)


def test_values_of_too_long_states_refused():
    assert call("vmoe_adamw_state_values", FAKE, FAKE, 1, 1 << 36, FAKE, 0, None) == UNS
