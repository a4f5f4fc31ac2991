"""Cases of the head's losses, their reference in float64 and the bounds of the tests.

U = 2^-24 is half a step of f32, UB = 2^-8 of bf16. Bounds, by row t and class c:
- z: d products and sums and the bias: ez = (d + 4) U (sum |x w| + |b|).
- lse: it moves by at most the largest ez of its row. An exponential's argument is off
  by 3 U (|z| + |m|), itself by 2 U; at most 64 terms a lane, 2 levels, a step a strip
  and wave, 8 waves: elf = max ez + U (90 + strips / 8 + 6 zmax), zmax = max |z| + 1.
- p = exp(z - lse): relative ep = ez + elf + U (8 + 6 zmax).
- q: arguments u off by 3 U |u|, the sum by 16 U: eq = U (24 + 4 max |u|).
- rates (weight, sum over rows in double, rounded; a product and a quotient): 6 U.
- dz: g p (ep + 6 U) + h p_T (ep_T + 6 U) + h Q (eq + (K + 8) U) at targets, and, in
  bf16, a rounding UB |dz|; ep_T from ez / T and so on.
- dx, dW, db: those errors through |W| and |x|, as many sums as there are terms (U
  each), and a rounding.
"""
import dataclasses
import math

import torch

from paper_2608_16188_amd import vmoe_head as H

from .train_common import TORCH, U, UB

DTYPES = {"f32": H.VMOE_F32, "bf16": H.VMOE_BF16}


@dataclasses.dataclass
class Case:
    n: int
    d: int
    v: int
    k: int = 0
    t: float = 1.0
    dtype: str = "bf16"
    bias: bool = True
    labels: bool = True
    weighted: bool = False
    ignored: float = 0.0
    missing: float = 0.0
    reduction: int = H.VMOE_REDUCE_MEAN
    seed: int = 1

    def shape(self):
        return H.make_head_shape(self.n, self.d, self.v, DTYPES[self.dtype], n_teacher=self.k,
                                 temperature=self.t, reduction=self.reduction)


W1, W2 = 0.7, 0.4  # w_label, w_teacher


class Data:
    """Inputs on the GPU (rows left out are spoilt only in what `run` hands over)."""

    def __init__(self, c: Case):
        g = torch.Generator(device="cuda").manual_seed(c.seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        rand = lambda *s: torch.rand(*s, device="cuda", generator=g)  # noqa: E731
        whole = lambda hi, *s: torch.randint(0, hi, s, device="cuda", generator=g)  # noqa: E731
        self.case, act = c, TORCH[c.dtype]
        w = randn(c.v, c.d) / math.sqrt(c.d)
        label = whole(c.v, c.n)
        self.x = (randn(c.n, c.d) + 10 * rand(c.n, 1) * w[label]).to(act)
        self.weight = w.to(act)
        self.bias = (0.5 * randn(c.v)).to(act) if c.bias else None
        out = rand(c.n) < c.ignored
        # (some rows keep a teacher without a label)
        no_label = out | (rand(c.n) < (0.2 if c.k and c.ignored else 0.0))
        odd = torch.tensor([-100, -1, c.v, 2 ** 31 - 1, -2 ** 31], device="cuda")[whole(5, c.n)]
        self.labels = torch.where(no_label, odd, label).to(torch.int32) if c.labels else None
        self.idx = self.logits = None
        if c.k:
            idx = whole(c.v, c.n, c.k)  # classes may come twice
            idx[:, 0] = torch.where(rand(c.n) < 0.7, label, idx[:, 0])
            gone = (rand(c.n, c.k) < c.missing) | out[:, None]
            self.idx = torch.where(gone, odd[:, None], idx).to(torch.int32)
            self.logits = 3 * randn(c.n, c.k)
        self.row_weight = 0.25 + rand(c.n) if c.weighted else None
        if c.weighted and c.n > 2:
            self.row_weight[whole(c.n, max(1, c.n // 8))] = 0.0

    def masks(self):
        c = self.case
        rw = torch.ones(c.n, device="cuda") if self.row_weight is None else self.row_weight
        none = torch.zeros(c.n, dtype=torch.bool, device="cuda")
        label = none if self.labels is None else (self.labels >= 0) & (self.labels < c.v) & (rw != 0)
        there = None if self.idx is None else (
            (self.idx >= 0) & (self.idx < c.v) & (self.logits != -math.inf) & (rw != 0)[:, None])
        taught = none if there is None else there.any(1)
        return rw.double(), label, there, taught

    def reference(self, w1=W1, w2=W2, bounds=True):
        """Values and bounds by output name."""
        c, T = self.case, self.case.t
        rw, label, there, taught = self.masks()
        live = label | taught
        x = torch.where(live[:, None], self.x.double(), 0.0)
        W = self.weight.double()
        b = torch.zeros(c.v, dtype=torch.float64, device="cuda") if self.bias is None \
            else self.bias.double()
        z = torch.mm(x, W.T) + b
        mag = torch.mm(x.abs(), W.abs().T) + b.abs()
        ez = (c.d + 4) * U * mag
        ezm = ez.amax(1)
        zmax = z.abs().amax(1) + 1
        strips = 2 * math.ceil(c.v / 128)
        acc = 90 + strips / 8
        lse = torch.logsumexp(z, 1)
        elf = ezm + U * (acc + 6 * zmax)
        a = torch.zeros(c.n, dtype=torch.float64, device="cuda")
        ea, bt, eb = a.clone(), a.clone(), a.clone()
        s1, s2 = (rw * label).sum(), (rw * taught).sum()
        mean = c.reduction == H.VMOE_REDUCE_MEAN
        g = w1 * rw * label / (s1 if mean and s1 != 0 else 1.0)
        h = w2 * T * rw * taught / (s2 if mean and s2 != 0 else 1.0)
        rows = torch.arange(c.n, device="cuda")
        p = torch.exp(z - lse[:, None])
        dz = g[:, None] * p
        ep = ezm + elf + U * (14 + 6 * zmax)
        edz = dz.abs() * ep[:, None]
        if self.labels is not None and c.n:
            y = torch.where(label, self.labels, 0).long()
            zl = z[rows, y]
            a = torch.where(label, lse - zl, 0.0)
            ea = torch.where(label, elf + ezm + 4 * U * zmax, 0.0)
            dz[rows, y] -= g
            edz[rows, y] += 8 * U * g.abs()
        if there is not None and c.n:
            y = torch.where(there, self.idx, 0).long()
            t = torch.where(there, self.logits.double(), -1e30) / T
            t = torch.where(taught[:, None], t, 0.0)
            lq = torch.log_softmax(t, 1)
            q = lq.exp() * there
            zt = z.gather(1, y) / T
            lse_t = torch.logsumexp(z / T, 1)
            elt = ezm / T + U * (acc + 6 * zmax / min(T, 1))
            kl = torch.where(there & (q != 0), q * (lq - zt), 0.0).sum(1) + lse_t
            u = torch.where(there & (q > 1e-40), (t - t.amax(1, keepdim=True)).abs(), 0.0).amax(1)
            eq = U * (24 + 4 * u)
            terms = torch.where(there & (q != 0), q * (lq.abs() + zt.abs()), 0.0).sum(1)
            bt = torch.where(taught, T * T * kl, 0.0)
            eb = torch.where(taught, T * T * ((eq + 24 * U) * terms + eq + 12 * U + ezm / T + elt
                                              + 4 * U * (terms + lse_t.abs())), 0.0)
            pt = torch.exp(z / T - lse_t[:, None])
            dense = h[:, None] * pt
            ept = ezm / T + elt + U * (14 + 6 * zmax / min(T, 1))
            dz += dense
            edz += dense.abs() * ept[:, None]
            dz.scatter_add_(1, y, -h[:, None] * q)
            edz.scatter_add_(1, y, (h.abs() * (eq + (c.k + 8) * U))[:, None] * q)
            del pt, dense
        del p
        ref = dict(losses=torch.stack([
            (rw * a).sum() / (s1 if mean and s1 != 0 else 1.0),
            (rw * bt).sum() / (s2 if mean and s2 != 0 else 1.0), s1, s2]),
            row_losses=torch.stack([a, bt], 1))
        if c.dtype == "bf16":
            edz += UB * (dz.abs() + edz)
        ref["dx"] = torch.where(live[:, None], torch.mm(dz, W), 0.0)
        ref["dweight"] = torch.mm(dz.T, x)
        ref["dbias"] = dz.sum(0)
        if not bounds:
            return ref
        un = UB if c.dtype == "bf16" else U
        one = lambda r: 1.01 * un * r.abs()  # noqa: E731
        size = dz.abs() + edz
        rel = 8 * U
        bound = dict(row_losses=torch.stack([ea, eb], 1) * 1.01 + 4 * U * ref["row_losses"].abs())
        e1 = (rw.abs() * (ea + rel * a.abs())).sum() / (s1 if mean and s1 != 0 else 1.0)
        e2 = (rw.abs() * (eb + rel * bt.abs())).sum() / (s2 if mean and s2 != 0 else 1.0)
        bound["losses"] = torch.stack([e1.abs(), e2.abs(), 2 * U * s1.abs(), 2 * U * s2.abs()])
        # Where a product is smaller than f32's least normal number it may be lost.
        tiny = 2.0 ** -126
        bound["dx"] = one(ref["dx"]) + (1 + un) * (
            torch.mm(edz, W.abs()) + (c.v + 80) * U * torch.mm(size, W.abs())) + tiny
        bound["dweight"] = one(ref["dweight"]) + (1 + un) * (
            torch.mm(edz.T, x.abs()) + (c.n + 80) * U * torch.mm(size.T, x.abs())) + tiny
        bound["dbias"] = one(ref["dbias"]) + (1 + un) * (
            edz.sum(0) + (c.n + 80) * U * size.sum(0)) + tiny
        return ref, bound

    def run(self, want=("dx", "dweight", "dbias"), w1=W1, w2=W2, spoil=True, stream=None,
            row_losses=True):
        """The library's outputs; what left-out rows and entries hold is not to matter."""
        c, s = self.case, self.case.shape()
        act = TORCH[c.dtype]
        rw, label, there, taught = self.masks()
        x, idx, logits = self.x.clone(), self.idx, self.logits
        if spoil and c.n:
            x[~(label | taught)] = float("nan")
            if there is not None:
                logits = torch.where(there | (logits == -math.inf), logits, float("nan"))
        pad = lambda t: t if t is None or t.numel() else torch.zeros(  # noqa: E731
            16, dtype=t.dtype, device="cuda")
        nan = lambda dt, *sh: torch.full(sh, float("nan"), dtype=dt, device="cuda")  # noqa: E731
        junk = lambda k: torch.full((max(k, 16),), 0xFF, dtype=torch.uint8,  # noqa: E731
                                    device="cuda")
        o = dict(losses=nan(torch.float32, 4),
                 row_losses=nan(torch.float32, max(c.n, 8), 2) if row_losses else None)
        saved = junk(H.vmoe_head_loss_saved_bytes(s))
        fwd, bwd = (junk(f(s)) for f in (H.vmoe_head_loss_fwd_workspace_bytes,
                                         H.vmoe_head_loss_bwd_workspace_bytes))
        H.vmoe_head_loss_fwd(s, pad(x), self.weight, self.bias, pad(self.labels), pad(idx),
                             pad(logits), pad(self.row_weight), o["losses"], o["row_losses"],
                             saved, fwd, stream)
        grads = dict(dx=nan(act, max(c.n, 8), c.d), dweight=nan(act, c.v, c.d),
                     dbias=nan(act, max(c.v, 8)))
        grads = {k: grads[k] for k in want}
        if want:
            H.vmoe_head_loss_bwd(s, self.weight, saved, w1, w2, grads.get("dx"),
                                 grads.get("dweight"), grads.get("dbias"), bwd, stream)
        torch.cuda.synchronize()
        o.update(grads)
        self.saved = saved
        # (what lies behind the last row stays as it was)
        for k, m in (("row_losses", c.n), ("dx", c.n), ("dbias", c.v)):
            if o.get(k) is not None:
                assert torch.isnan(o[k][m:]).all(), k
                o[k] = o[k][:m]
        return {k: t for k, t in o.items() if t is not None}
