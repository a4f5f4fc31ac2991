"""What a training step learns from: a head over many classes with its losses, as cases that can be timed and compared.

Two operators over the rows of x [N, d] and a head's weight [V, d]: softmax cross
entropy against labels, and distillation from a teacher's top logits, each with
its gradients in x, weight and bias, separately and together. `run` computes them
through the library where `own` is true and in elementary torch operations where
it is not; `exact` is the definition in 64 bits. Rows are the tokens of the
benchmark's workloads, of neighbouring batches, or single images.
"""
from __future__ import annotations

import math

import torch

own = False  # True: through the library's entry points

DEV = "cuda"


# ------------------------------------------------------------------ cases

def _case(name, rows, d, classes, **more):
    """pass: train (loss and gradients) | eval (loss alone) | frozen (no gradient of
    the head). top: entries of the teacher's list, 0 without a teacher. ignored:
    share of rows without label and teacher. missing: of the teacher's entries."""
    c = dict(name=name, rows=rows, d=d, classes=classes, dtype="bf16", bias=False, labels=True,
             top=0, temperature=1.0, ignored=0.0, missing=0.0, weighted=False)
    c["pass"] = "train"
    c.update(more)
    return c


def listed():
    return [
        # One image's class token through a classifier: launch latency.
        _case("labels_one_image", 1, 768, 1000, bias=True),
        # The small f32 layer's tokens, of which only the four class tokens have
        # a label.
        _case("labels_tiny_f32", 788, 192, 1000, dtype="f32", bias=True, ignored=0.995),
        # Class tokens of one batch of images and a large set of classes: the
        # head's weights are most of what is moved.
        _case("labels_class_tokens", 64, 1024, 21841, bias=True),
        # Every token of a ViT-B/16 batch against an odd vocabulary.
        _case("labels_vitb16_tokens", 6304, 768, 32003),
        # Evaluation: the loss alone over a wider vocabulary.
        _case("labels_eval", 4616, 1024, 50021, **{"pass": "eval"}),
        # The headline batch of tokens, a quarter of them padding, weighted rows.
        _case("labels_vitl16_tokens", 36928, 1024, 32000, ignored=0.25, weighted=True),
        # A few images with labels and a teacher's ten best classes.
        _case("teacher_few_images", 16, 768, 1000, bias=True, top=10, temperature=2.0),
        # Tokens of a ViT-B/16 batch with labels and a teacher's 32 best.
        _case("teacher_vitb16_tokens", 6304, 768, 32003, top=32, temperature=2.0),
        # A teacher alone, a wide model and a large odd vocabulary.
        _case("teacher_wide", 2047, 4096, 65537, bias=True, labels=False, top=64),
        # A small f32 model, ragged: padding, lists of unequal length.
        _case("teacher_ragged_f32", 1171, 328, 5003, dtype="f32", bias=True, top=100,
              temperature=4.0, ignored=0.4, missing=0.3, weighted=True),
        # A frozen head: only the gradient of the tokens is wanted.
        _case("teacher_frozen_head", 6304, 1024, 16384, top=16, temperature=1.5,
              **{"pass": "frozen"}),
    ]


_LARGEST = 36928 * 32000 * 1024


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the listed ranges: 1 to 40 000 rows, widths 64 to 4096 and
    10 to 130 000 classes, lists of 1 to 200."""
    while True:
        rows, d, classes = _log(rng, 1, 40000), 8 * _log(rng, 8, 512), _log(rng, 10, 130000)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        size = rows * d * classes
        if size > _LARGEST * (3 / 4 if dtype == "bf16" else 1 / 16) or rows * classes > 1.2e9:
            continue
        if rows * classes < 20000 and rng.random() < 0.7:
            continue  # few of the very smallest
        top = rng.choice([0, 0, 1]) and min(classes, _log(rng, 1, 200))
        c = _case("", rows, d, classes, dtype=dtype, bias=rng.random() < 0.5, top=top,
                  labels=top == 0 or rng.random() < 0.6,
                  temperature=rng.choice([1.0, 1.5, 2.0, 4.0]) if top else 1.0,
                  ignored=rng.choice([0.0, 0.0, 0.1, 0.5, 0.9]) if rows > 8 else 0.0,
                  missing=rng.choice([0.0, 0.3]) if top > 4 else 0.0,
                  weighted=rng.random() < 0.3,
                  **{"pass": rng.choice(["train", "train", "train", "eval", "frozen"])})
        del c["name"]
        return c


def _t(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def work(c):
    size = 2 if c["dtype"] == "bf16" else 4
    rows = max(1, round(c["rows"] * (1 - c["ignored"])))
    x, w = rows * c["d"] * size, c["classes"] * (c["d"] + (1 if c["bias"] else 0)) * size
    small = rows * (8 * c["top"] + 4 * c["labels"]) + 8 * c["rows"]
    products = dict(eval=1, frozen=2, train=3)[c["pass"]]
    out = dict(eval=0, frozen=c["rows"] * c["d"] * size,
               train=c["rows"] * c["d"] * size + w)[c["pass"]]
    return dict(bytes=x + w + small + out, flops=2 * products * rows * c["d"] * c["classes"])


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    c, n, d, V, K = case, case["rows"], case["d"], case["classes"], case["top"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    rand = lambda *s: torch.rand(*s, device=DEV, generator=g)  # noqa: E731
    draw_class = lambda *s: torch.randint(0, V, s, device=DEV, generator=g)  # noqa: E731
    s = dict(case=c)
    weight = randn(V, d) / math.sqrt(d)
    s["weight"] = weight.to(_t(c["dtype"]))
    s["bias"] = (0.5 * randn(V)).to(_t(c["dtype"])) if c["bias"] else None
    label = draw_class(n)
    # normalised tokens that lean towards their class: some rows are unsure, some
    # almost certain
    s["x"] = (randn(n, d) + 14 * rand(n, 1) * weight[label]).to(_t(c["dtype"]))
    live = rand(n) >= c["ignored"]
    live[0] = True
    s["labels"] = torch.where(live, label, -100).to(torch.int32) if c["labels"] else None
    s["teacher_idx"] = s["teacher_logits"] = None
    if K:
        # distinct classes, the label's mostly first; logits that fall with the rank
        step = torch.randint(1, max(2, V // K), (n, K), device=DEV, generator=g)
        idx = (torch.where(rand(n) < 0.9, label, draw_class(n))[:, None] + step.cumsum(1)
               - step[:, :1]) % V
        fall = torch.arange(1, K + 1, device=DEV).float().log()
        there = (rand(n, K) >= c["missing"]) & live[:, None]
        there[:, 0] |= live
        s["teacher_idx"] = torch.where(there, idx, -1).to(torch.int32)
        s["teacher_logits"] = 9 + 2 * randn(n, 1) - 2.5 * fall + 0.3 * randn(n, K)
    s["row_weight"] = 0.5 + rand(n) if c["weighted"] else None
    s["w_label"], s["w_teacher"] = (0.4 if K else 1.0), 0.6
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------ through the library

def _handles(s):
    """The shape, buffers and outputs that a program makes once."""
    from paper_2608_16188_amd import vmoe_head as H
    c, n, d, V = s["case"], s["case"]["rows"], s["case"]["d"], s["case"]["classes"]
    dt = H.VMOE_BF16 if c["dtype"] == "bf16" else H.VMOE_F32
    s["shape"] = sh = H.make_head_shape(n, d, V, dt, n_teacher=c["top"],
                                        temperature=c["temperature"])
    new = lambda dtype, *shape: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    bytes_ = lambda k: new(torch.uint8, max(k, 16))  # noqa: E731
    s["saved"] = bytes_(H.vmoe_head_loss_saved_bytes(sh))
    s["fwd_ws"] = bytes_(H.vmoe_head_loss_fwd_workspace_bytes(sh))
    s["out"] = dict(losses=new(torch.float32, 4), row_losses=new(torch.float32, n, 2))
    if c["pass"] != "eval":
        s["bwd_ws"] = bytes_(H.vmoe_head_loss_bwd_workspace_bytes(sh))
        s["out"]["dx"] = new(_t(c["dtype"]), n, d)
        if c["pass"] == "train":
            s["out"]["dweight"] = new(_t(c["dtype"]), V, d)
            if c["bias"]:
                s["out"]["dbias"] = new(_t(c["dtype"]), V)


def _run_own(s):
    from paper_2608_16188_amd import vmoe_head as H
    o = s["out"]
    H.vmoe_head_loss_fwd(s["shape"], s["x"], s["weight"], s["bias"], s["labels"], s["teacher_idx"],
                         s["teacher_logits"], s["row_weight"], o["losses"], o["row_losses"],
                         s["saved"], s["fwd_ws"])
    if s["case"]["pass"] != "eval":
        H.vmoe_head_loss_bwd(s["shape"], s["weight"], s["saved"], s["w_label"],
                             s["w_teacher"], o["dx"], o.get("dweight"), o.get("dbias"),
                             s["bwd_ws"])
    return dict(o)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ plain form

def _softmax(z):
    """Probabilities and the logarithm of their sum of exponentials, a row each."""
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    return e / total, (top + torch.log(total))[:, 0]


def _mean(loss, weight):
    total = weight.double().sum()
    safe = torch.where(total == 0, 1.0, total)
    return (loss.double() * weight).sum() / safe, total, weight / safe.float()


def _run_plain(s):
    c, V = s["case"], s["case"]["classes"]
    T = c["temperature"]
    x, w = s["x"].float(), s["weight"].float()
    n = x.shape[0]
    z = torch.matmul(x, w.T)
    if s["bias"] is not None:
        z = z + s["bias"].float()
    rw = torch.ones(n, device=DEV) if s["row_weight"] is None else s["row_weight"]
    zero = torch.zeros(n, device=DEV)
    loss1 = loss2 = weight1 = weight2 = zero
    grad = None
    if s["labels"] is not None:
        there = (s["labels"] >= 0) & (s["labels"] < V)
        label = torch.where(there, s["labels"], 0).long()[:, None]
        p, lse = _softmax(z)
        loss1 = torch.where(there, lse - z.gather(1, label)[:, 0], 0.0)
        weight1 = torch.where(there, rw, 0.0)
        mean1, sum1, rate = _mean(loss1, weight1)
        if c["pass"] != "eval":
            rate = (s["w_label"] * rate)[:, None]
            grad = (p * rate).scatter_add_(1, label, -rate)
    else:
        mean1 = sum1 = zero.sum()
    if s["teacher_idx"] is not None:
        there = (s["teacher_idx"] >= 0) & (s["teacher_idx"] < V)
        idx = torch.where(there, s["teacher_idx"], 0).long()
        t = torch.where(there, s["teacher_logits"] / T, -math.inf)
        taught = there.any(1)
        q, lq = _softmax(torch.where(taught[:, None], t, 0.0))
        q = torch.where(there, q, 0.0)
        p, lse = _softmax(z / T)
        terms = torch.where(there, q * (t - lq[:, None] - z.gather(1, idx) / T), 0.0)
        loss2 = torch.where(taught, T * T * (terms.sum(1) + lse), 0.0)
        weight2 = torch.where(taught, rw, 0.0)
        mean2, sum2, rate = _mean(loss2, weight2)
        if c["pass"] != "eval":
            rate = (s["w_teacher"] * T * rate)[:, None]
            more = (p * rate).scatter_add_(1, idx, -q * rate)
            grad = more if grad is None else grad + more
    else:
        mean2 = sum2 = zero.sum()
    out = dict(losses=torch.stack([v.float() for v in (mean1, mean2, sum1, sum2)]),
               row_losses=torch.stack([loss1, loss2], 1))
    act = _t(c["dtype"])
    if c["pass"] != "eval":
        out["dx"] = torch.matmul(grad, w).to(act)
        if c["pass"] == "train":
            out["dweight"] = torch.matmul(grad.T, x).to(act)
            if c["bias"]:
                out["dbias"] = grad.sum(0).to(act)
    return out


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    """Loss of every row, then the derivative of w_label mean1 + w_teacher mean2, a
    slice of rows at a time."""
    s = prepare(case, seed)
    c, V, T = case, case["classes"], case["temperature"]
    n, w = case["rows"], s["weight"].double()
    b = torch.zeros(V, dtype=torch.float64, device=DEV) if s["bias"] is None \
        else s["bias"].double()
    rw = torch.ones(n, dtype=torch.float64, device=DEV) if s["row_weight"] is None \
        else s["row_weight"].double()
    none = torch.zeros(n, dtype=torch.bool, device=DEV)
    labelled = none if s["labels"] is None else (s["labels"] >= 0) & (s["labels"] < V)
    listed_ = None if s["teacher_idx"] is None else (s["teacher_idx"] >= 0) & (s["teacher_idx"] < V)
    taught = none if listed_ is None else listed_.any(1)
    w1, w2 = rw * labelled, rw * taught
    sums = [w1.sum(), w2.sum()]
    rows = torch.zeros(n, 2, dtype=torch.float64, device=DEV)
    dx = torch.zeros(n, case["d"], dtype=torch.float64, device=DEV)
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    step = max(1, int(2.5e8) // V)
    for at in range(0, n, step):
        part = slice(at, min(n, at + step))
        k = torch.arange(part.stop - part.start, device=DEV)
        x = s["x"][part].double()
        z = torch.addmm(b, x, w.T)
        dz = torch.zeros_like(z)
        if s["labels"] is not None and sums[0] != 0:
            lp = torch.log_softmax(z, 1)
            y = s["labels"][part].long().clamp(0, V - 1)
            rows[part, 0] = -lp[k, y] * labelled[part]
            rate = s["w_label"] * w1[part] / sums[0]
            dz += lp.exp_() * rate[:, None]
            dz[k, y] -= rate
        if listed_ is not None and sums[1] != 0:
            lp = torch.log_softmax(z / T, 1)
            y = s["teacher_idx"][part].long().clamp(0, V - 1)
            t = s["teacher_logits"][part].double() / T
            t = torch.where(listed_[part], t, -1e300)
            lq = torch.log_softmax(t, 1)
            q = lq.exp() * listed_[part]
            kl = (q * (lq - lp.gather(1, y))).sum(1)
            rows[part, 1] = T ** 2 * kl * taught[part]
            rate = s["w_teacher"] * T * (w2[part] / sums[1])
            dz += lp.exp_() * rate[:, None]
            dz.scatter_add_(1, y, -q * rate[:, None])
        if c["pass"] != "eval":
            dx[part] = torch.mm(dz, w)
        if c["pass"] == "train":
            dw += torch.mm(dz.T, x)
            db += dz.sum(0)
    means = [(rows[:, i] * (w1, w2)[i]).sum() / sums[i] if sums[i] != 0 else sums[i]
             for i in range(2)]
    out = dict(losses=torch.stack(means + sums), row_losses=rows)
    if c["pass"] != "eval":
        out["dx"] = dx
        if c["pass"] == "train":
            out["dweight"] = dw
            if c["bias"]:
                out["dbias"] = db
    return out
