"""Host-side checks of vmoe_head.h's calls (no GPU, nothing is launched): exported
symbols, sizes of buffers, refusals before anything is enqueued, the binding's own."""
import ctypes
import math
import re
import subprocess

import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_head as H
from paper_2608_16188_amd import workloads as W
from paper_2608_16188_amd.block import SparseBlock

from .other_gpu import Elsewhere

FAKE = 0x10000  # 16-byte aligned, never dereferenced
BAD, UNS, WS = V.VMOE_ERR_INVALID_ARG, V.VMOE_ERR_UNSUPPORTED, V.VMOE_ERR_WORKSPACE
P, Z, I32, F = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
SIGNATURES = {"vmoe_head_loss_fwd": (I32, [P] * 12 + [Z, P]),
              "vmoe_head_loss_bwd": (I32, [P] * 3 + [F] * 2 + [P] * 4 + [Z, P])}
SIZES = (H.vmoe_head_loss_saved_bytes, H.vmoe_head_loss_fwd_workspace_bytes,
         H.vmoe_head_loss_bwd_workspace_bytes)


def call(name, *args):
    f = ctypes.CDLL(V.LIB_PATH)[name]  # a function object of its own
    f.restype, f.argtypes = SIGNATURES[name]
    return f(*args)


def _shape(**kw):
    base = dict(n_rows=8, d_model=64, n_classes=100, dtype=V.VMOE_BF16)
    base.update(kw)
    sizes = [base.pop(k) for k in ("n_rows", "d_model", "n_classes", "dtype")]
    return H.make_head_shape(*sizes, **base)


def test_declared_symbols_are_exported():
    text = open(H.HEADER).read()
    declared = set(re.findall(r"^\s*[\w\s\*]+?\b(vmoe_\w+)\s*\(", text, re.M))
    assert declared == {f"vmoe_head_loss_{k}" for k in (
        "saved_bytes", "fwd_workspace_bytes", "bwd_workspace_bytes", "fwd", "bwd")}, declared
    out = subprocess.check_output(["nm", "-D", "--defined-only", V.LIB_PATH], text=True)
    assert declared <= {line.split()[-1] for line in out.splitlines() if line.strip()}
    assert all(hasattr(H, s) for s in declared)


REFUSED = [
    (dict(n_rows=-1), BAD), (dict(d_model=12), BAD), (dict(d_model=0), BAD),
    (dict(d_model=-8), BAD), (dict(n_classes=0), BAD), (dict(n_classes=-5), BAD),
    (dict(n_teacher=-1), BAD), (dict(n_teacher=257), BAD), (dict(dtype=2), BAD),
    (dict(dtype=-1), BAD), (dict(reduction=2), BAD), (dict(reduction=-1), BAD),
    (dict(temperature=0.0), BAD), (dict(temperature=-1.0), BAD),
    (dict(temperature=math.nan), BAD), (dict(temperature=math.inf), BAD),
    (dict(temperature=2.0 ** -11), BAD), (dict(temperature=1025.0), BAD),
    (dict(n_rows=2 ** 21 + 1, d_model=8, n_classes=1), UNS),
    (dict(n_rows=2 ** 20 + 1, d_model=8, n_classes=1, dtype=V.VMOE_F32), UNS),
    (dict(n_classes=2 ** 21 + 1, n_rows=1), UNS), (dict(d_model=65544, n_rows=1), UNS),
    (dict(n_rows=2 ** 20, d_model=1024), UNS),
    (dict(n_rows=2 ** 19, d_model=1024, dtype=V.VMOE_F32), UNS),
    (dict(n_rows=2 ** 16, n_classes=2 ** 20), UNS),
]


@pytest.mark.parametrize("kw, status", REFUSED)
def test_shapes_refused(kw, status):
    s = _shape(**kw)
    assert all(f(s) == 0 for f in SIZES)
    ref = ctypes.addressof(s)
    big = 1 << 60
    labels = FAKE if s.n_teacher == 0 else None
    assert call("vmoe_head_loss_fwd", ref, FAKE, FAKE, None, labels, None, None, None, FAKE, None,
                FAKE, FAKE, big, None) == status
    assert call("vmoe_head_loss_bwd", ref, FAKE, FAKE, 1.0, 1.0, FAKE, FAKE, FAKE, FAKE, big,
                None) == status
    s.reserved = 1
    assert call("vmoe_head_loss_bwd", ref, FAKE, FAKE, 1.0, 1.0, FAKE, FAKE, FAKE, FAKE, big,
                None) == BAD


def test_no_shape_and_reserved_refused():
    s = _shape()
    s.reserved = 7
    for ref in (None, ctypes.addressof(s)):
        assert call("vmoe_head_loss_fwd", ref, FAKE, FAKE, None, FAKE, None, None, None, FAKE,
                    None, FAKE, FAKE, 1 << 60, None) == BAD
        assert call("vmoe_head_loss_bwd", ref, FAKE, FAKE, 1.0, 1.0, FAKE, None, None, FAKE,
                    1 << 60, None) == BAD


def _fwd(s, **kw):
    a = dict(x=FAKE, weight=FAKE, bias=None, labels=FAKE, idx=None, logits=None, row_weight=None,
             losses=FAKE, row_losses=None, saved=FAKE, ws=FAKE,
             bytes=H.vmoe_head_loss_fwd_workspace_bytes(s))
    a.update(kw)
    return call("vmoe_head_loss_fwd", ctypes.addressof(s), *a.values(), None)


ODD = FAKE + 8


@pytest.mark.parametrize("k, kw, status", [
    (0, dict(x=None), BAD), (0, dict(weight=None), BAD), (0, dict(losses=None), BAD),
    (0, dict(saved=None), BAD), (0, dict(labels=None), BAD), (0, dict(idx=FAKE), BAD),
    (0, dict(logits=FAKE), BAD), (3, dict(), BAD), (3, dict(idx=FAKE), BAD),
    (3, dict(logits=FAKE), BAD), (3, dict(idx=FAKE, logits=ODD), BAD),
    (3, dict(idx=ODD, logits=FAKE), BAD), (0, dict(x=ODD), BAD), (0, dict(weight=ODD), BAD),
    (0, dict(bias=ODD), BAD), (0, dict(labels=ODD), BAD), (0, dict(row_weight=ODD), BAD),
    (0, dict(losses=ODD), BAD), (0, dict(row_losses=ODD), BAD), (0, dict(saved=ODD), BAD),
    (0, dict(ws=None), WS), (0, dict(ws=ODD), WS), (0, dict(bytes=0), WS),
])
def test_arguments_of_the_forward_refused(k, kw, status):
    assert _fwd(_shape(n_teacher=k), **kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(weight=None), BAD), (dict(saved=None), BAD), (dict(w1=math.nan), BAD),
    (dict(w2=math.inf), BAD), (dict(dx=None, dw=None, db=None), BAD), (dict(dx=ODD), BAD),
    (dict(dw=ODD), BAD), (dict(db=ODD), BAD), (dict(weight=ODD), BAD), (dict(saved=ODD), BAD),
    (dict(ws=None), WS), (dict(ws=ODD), WS), (dict(bytes=255), WS),
])
def test_arguments_of_the_backward_refused(kw, status):
    a = dict(weight=FAKE, saved=FAKE, w1=1.0, w2=1.0, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE,
             bytes=H.vmoe_head_loss_bwd_workspace_bytes(_shape()))
    a.update(kw)
    assert call("vmoe_head_loss_bwd", ctypes.addressof(_shape()), *a.values(), None) == status


def test_a_teachers_weight_that_overflows_refused():
    s = _shape(n_teacher=2, temperature=1024.0)
    assert call("vmoe_head_loss_bwd", ctypes.addressof(s), FAKE, FAKE, 1.0, 1e36, FAKE, FAKE, FAKE,
                FAKE, H.vmoe_head_loss_bwd_workspace_bytes(s), None) == BAD


@pytest.mark.parametrize("n, d, v, k", [
    (0, 8, 1, 0), (1, 8, 1, 256), (64, 768, 1000, 10), (65, 768, 1000, 10), (6304, 768, 50000, 0),
    (36928, 1024, 32000, 64), (2 ** 21, 8, 2 ** 14, 0), (1, 65536, 2 ** 21, 0),
    (2 ** 15, 256, 2 ** 20, 0),
])
@pytest.mark.parametrize("dtype", [V.VMOE_F32, V.VMOE_BF16])
def test_buffers_do_not_grow_with_the_logits(n, d, v, k, dtype):
    """saved: the rows, and few logits; forward: a few numbers a row and strip of classes;
    backward: 1 GiB of dz, f32 sums of dx in up to 64 ranges and of a piece's dweight in
    up to 16 (only where either has few tiles)."""
    s = _shape(n_rows=n, d_model=d, n_classes=v, n_teacher=k, dtype=dtype)
    size = 2 if dtype == V.VMOE_BF16 else 4
    if n * d * size >= 2 ** 31 or n * size > 2 ** 22:
        assert SIZES[0](s) == 0
        return
    saved, fwd, bwd = (f(s) for f in SIZES)
    most = 2 ** 22 if dtype == V.VMOE_BF16 else 2 ** 26
    logits = 4 * n * (v + 31) if n <= 64 or (n + 63) * v <= most else 0
    assert n * d * size < saved <= n * (d * size + 32 + 12 * (k + 1)) + 4 * v + logits + 8192
    strips = v / 32 + 4
    assert 0 < fwd <= n * (12 * strips + 4 * k) + 4 * (n / 64 + 1) * (v / 128 + 1) + n + 8192
    assert 0 < bwd <= 2 ** 30 + 512 * n * size + (64 * 4 * n * d if n < 4096 else 2 ** 31) \
        + 2 ** 31 + 4 * n * d + 8192


def test_the_binding_names_what_it_refuses():
    s = _shape()
    c = lambda *sh, dt=torch.bfloat16: torch.zeros(*sh, dtype=dt)  # noqa: E731
    a = dict(x=None, weight=None, bias=None, labels=None, teacher_idx=None, teacher_logits=None,
             row_weight=None, losses=None, row_losses=None, saved=None, workspace=None)
    g = lambda *sh, dt=torch.bfloat16: Elsewhere(0, *sh, dtype=dt)  # noqa: E731
    for name, bad in (("x", c(8, 64)), ("x", g(8, 63)), ("weight", g(99, 64)),
                      ("weight", g(100, 64, dt=torch.float32)), ("bias", g(99)),
                      ("labels", g(8, dt=torch.int64)), ("labels", g(7, dt=torch.int32)),
                      ("row_weight", g(8)), ("losses", g(3, dt=torch.float32)),
                      ("row_losses", g(8, dt=torch.float32)), ("saved", g(64, dt=torch.uint8)),
                      ("saved", g(1 << 20, dt=torch.int8))):
        with pytest.raises(ValueError, match=f"^{name}: a contiguous .* is wanted"):
            H.vmoe_head_loss_fwd(s, **{**a, name: bad}, stream=0)
    with pytest.raises(ValueError, match="^weight: a tensor on cuda:0 is wanted.*cuda:1"):
        H.vmoe_head_loss_fwd(s, **{**a, "x": g(8, 64),
                                   "weight": Elsewhere(1, 100, 64, dtype=torch.bfloat16)},
                             stream=0)
    t = _shape(n_teacher=5)
    for name, bad in (("teacher_idx", g(8, 4, dt=torch.int32)),
                      ("teacher_idx", g(8, 5, dt=torch.int64)), ("teacher_logits", g(8, 5))):
        with pytest.raises(ValueError, match=f"^{name}: a contiguous"):
            H.vmoe_head_loss_fwd(t, **{**a, name: bad}, stream=0)
    b = dict(weight=None, saved=None, w_label=1.0, w_teacher=1.0, dx=None, dweight=None,
             dbias=None, workspace=None)
    for name, bad in (("dx", g(8, 64, dt=torch.float32)), ("dweight", g(100, 63)),
                      ("dbias", g(99)), ("saved", g(16, dt=torch.uint8))):
        with pytest.raises(ValueError, match=f"^{name}: a contiguous"):
            H.vmoe_head_loss_bwd(s, **{**b, name: bad}, stream=0)
    with pytest.raises(TypeError, match="a HeadShape is wanted"):
        H.vmoe_head_loss_bwd(V.make_shape(8, 1, 64, 64, 2, 1, 1.0, V.VMOE_F32), **b)
    with pytest.raises(TypeError):
        H.vmoe_head_loss_bwd(s, **{**b, "w_label": "much"}, stream=0)


@pytest.mark.parametrize("options", [dict(classes=-1), dict(teacher_top=4),
                                     dict(classes=10, teacher_top=-1),
                                     dict(classes=10, teacher_top=257)])
def test_options_of_the_block_refused(options):
    cfg = W.custom_config("refused", n_tokens=16, d_model=64, d_ff=64, n_experts=2, k=1,
                          capacity_factor=1.0)
    with pytest.raises(ValueError, match="^classes, teacher_top: "):
        SparseBlock(cfg, {}, **options)


@pytest.mark.parametrize("options", [["--teacher-top", "5"], ["--classes", "-1"],
                                     ["--classes", "4", "--teacher-top", "5"],
                                     ["--classes", "1000", "--teacher-top", "257"]])
def test_options_of_the_command_refused(options, monkeypatch, capsys):
    from paper_2608_16188_amd import block
    monkeypatch.setattr("sys.argv", ["block", *options])
    with pytest.raises(SystemExit) as e:
        block.main()
    assert e.value.code == 2 and "--teacher-top" in capsys.readouterr().err
