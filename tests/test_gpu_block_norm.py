"""Block norm on the GPU against a float64 form of its definition and, for the
backward, against autograd through that form and against differences of it.

Bounds are sums of roundings, U = 2^-24 each: a value of the chain passes fewer
than 100 (a lane adds at most 32 of a row's columns, the lanes and waves of a
team 6 + 16 more, a block's rows and the partial rows of a column at most 40 at
these sizes, and each term has some 20 of its own), against the sum of the
magnitudes that meet there; K = 128 of them are allowed. bf16 outputs add one
rounding."""
import numpy as np
import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

from .gpu_common import say
from .train_common import DTYPES, NORMS, TORCH, U, close, rounding, same_bits

pytestmark = pytest.mark.gpu
K = 128
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


class Case:
    """Inputs of one call on the CPU in float64 (exactly what the types hold)."""

    def __init__(self, n, d, dtype="bf16", stream=None, dh="f32", groups=1, pre="layer",
                 post="none", weights=True, bias=True, gate=True, drop=0.0, residual=1.0,
                 branch=1.0, block=True, up=True, seed=0, offset=0.3):
        self.n, self.d, self.groups, self.pre, self.post = n, d, groups, pre, post
        self.dtype, self.stream, self.dh_t = dtype, stream or dtype, "f32" if dtype == "f32" else dh
        self.residual, self.branch, self.block = residual, branch, block
        rng = np.random.default_rng(seed)
        draw = lambda t, *s: torch.from_numpy(rng.standard_normal(s)).to(TORCH[t]).double()  # noqa: E731
        self.x = (draw("f32", n, d) * 2 + offset).to(TORCH[self.stream]).double()
        self.y = (draw("f32", n, d) + offset).to(TORCH[dtype]).double() if block else None
        vec = lambda mean: (mean + 0.3 * draw("f32", d)).to(TORCH[dtype]).double()  # noqa: E731
        has_pre, has_post = pre != "none", post != "none" and block
        self.pre_w = vec(1.0) if has_pre and weights else None
        self.pre_b = vec(0.0) if has_pre and bias else None
        self.post_w = vec(1.0) if has_post and weights else None
        self.post_b = vec(0.0) if has_post and bias else None
        self.gate = (0.5 + 0.5 * draw("f32", groups, d)).to(TORCH[dtype]).double() \
            if gate and block else None
        self.row = None
        if drop and block:
            keep = torch.from_numpy((rng.random(n) >= drop).astype(np.float32))
            self.row = (keep / np.float32(1 - drop)).double()
        self.dx_out = draw(self.stream, n, d) if up else None
        self.dh = draw(self.dh_t, n, d) if has_pre else None

    def shape(self):
        return T.make_norm_shape(self.n, self.d, DTYPES[self.dtype], n_groups=self.groups,
                                 stream_dtype=DTYPES[self.stream], dh_dtype=DTYPES[self.dh_t],
                                 pre_norm=NORMS[self.pre], post_norm=NORMS[self.post], eps=EPS,
                                 residual_scale=self.residual, branch_scale=self.branch)

    # ------------------------------------------------------ float64
    def params(self):
        return {k: getattr(self, k) for k in ("pre_w", "pre_b", "post_w", "post_b", "gate")}

    def forward(self, x, y, p):
        """x_out, h and both [N, 2] statistics from the definition."""
        out = {}
        eps = float(np.float32(EPS))

        def norm(v, kind, w, b, key, on=None):
            mu = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
            r = 1 / torch.sqrt((v - mu).square().mean(1, keepdim=True) + eps)
            stats = torch.cat([mu, r], 1)
            out[key] = stats if on is None else torch.where(on[:, None], stats, 0.0)
            v = (v - mu) * r
            v = v * w if w is not None else v
            return v + b if b is not None else v

        if self.block:
            on = torch.ones(self.n, dtype=torch.bool) if self.row is None else self.row != 0
            if self.post != "none":
                y = norm(y, self.post, p["post_w"], p["post_b"], "post_stats", on)
            if p["gate"] is not None:
                y = y * p["gate"].repeat_interleave(max(self.n // self.groups, 1), 0)[:self.n]
            a = float(np.float32(self.branch))
            if self.row is not None:
                y = y * self.row[:, None]
            x = float(np.float32(self.residual)) * x + a * y
            out["x_out"] = x
        if self.pre != "none":
            out["h"] = norm(x, self.pre, p["pre_w"], p["pre_b"], "pre_stats")
        return out


def _dev(t, kind):
    """On the GPU in its type; an empty batch still hands over an allocation."""
    if t is None:
        return None
    if t.numel() == 0:
        t = torch.zeros(16)
    return t.to(TORCH[kind]).cuda().contiguous()


def _new(n, d, kind, fill=float("nan")):
    return torch.full((max(n, 1), d), fill, dtype=TORCH[kind], device="cuda")


def run_forward(c, spoil_dropped=False, stream=None, in_place=False):
    x = _dev(c.x, c.stream)
    y = _dev(c.y, c.dtype)
    if spoil_dropped:
        y[c.row.cuda() == 0] = float("nan")
    p = {k: _dev(v, c.dtype) for k, v in c.params().items()}
    o = dict(x_out=(x if in_place else _new(c.n, c.d, c.stream)) if c.block else None,
             h=_new(c.n, c.d, c.dtype) if c.pre != "none" else None,
             post_stats=_new(c.n, 2, "f32") if c.post != "none" and c.block else None,
             pre_stats=_new(c.n, 2, "f32") if c.pre != "none" else None)
    T.vmoe_block_norm_fwd(c.shape(), x, y, p["post_w"], p["post_b"], p["gate"], _dev(c.row, "f32"),
                          p["pre_w"], p["pre_b"], o["x_out"], o["h"], o["post_stats"],
                          o["pre_stats"], stream)
    torch.cuda.synchronize()
    return {k: v[:c.n] for k, v in o.items() if v is not None}


def run_backward(c, x_out, pre_stats, post_stats, spoil_dropped=False, in_place=False, skip=()):
    """At a given x_out (the stream's type) and statistics."""
    p = {k: _dev(v, c.dtype) for k, v in c.params().items()}
    y = _dev(c.y, c.dtype)
    if spoil_dropped:
        y[c.row.cuda() == 0] = float("inf")
    dx_out = _dev(c.dx_out, c.stream)
    o = dict(dx=dx_out if in_place else _new(c.n, c.d, c.stream),
             dy=(y if in_place else _new(c.n, c.d, c.dtype)) if c.block else None)
    for k, t in (("dpost_w", c.post_w), ("dpost_b", c.post_b), ("dgate", c.gate),
                 ("dpre_w", c.pre_w), ("dpre_b", c.pre_b)):
        rows = c.groups if k == "dgate" else 1
        o[k] = None if t is None or k in skip else _new(rows, c.d, "f32")
    s = c.shape()
    ws = torch.full((max(T.vmoe_block_norm_bwd_workspace_bytes(s), 16),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    T.vmoe_block_norm_bwd(s, dx_out, _dev(c.dh, c.dh_t), _dev(x_out, c.stream), y, p["post_w"],
                          p["post_b"], p["gate"], _dev(c.row, "f32"), p["pre_w"],
                          _dev(post_stats, "f32"), _dev(pre_stats, "f32"), o["dx"], o["dy"],
                          o["dpost_w"], o["dpost_b"], o["dgate"], o["dpre_w"], o["dpre_b"], ws)
    torch.cuda.synchronize()
    for k in ("dx", "dy"):
        if o[k] is not None:
            o[k] = o[k][:c.n]
    for k in ("dpost_w", "dpost_b", "dpre_w", "dpre_b"):
        if o[k] is not None:
            o[k] = o[k][0]
    return {k: v for k, v in o.items() if v is not None}


CASES = {
    # widths on both sides of every choice of waves a row, ends inside a lane's step
    "one_token": dict(n=1, d=8),
    "one_vector_f32": dict(n=3, d=8, dtype="f32", post="layer"),
    "d192_f32": dict(n=197, d=192, dtype="f32", post="rms", bias=False),
    "d504": dict(n=37, d=504, post="layer", drop=0.4),
    "d512_groups": dict(n=60, d=512, groups=5, post="rms", dh="bf16"),
    "d520": dict(n=41, d=520, pre="rms", bias=False),
    "d1000_stream": dict(n=65, d=1000, stream="f32", post="layer", drop=0.2),
    "d1024_scales": dict(n=130, d=1024, residual=0.75, branch=-1.5, drop=0.5),
    "d1032": dict(n=19, d=1032, post="layer", stream="f32", dh="bf16"),
    "d2048_f32": dict(n=9, d=2048, dtype="f32", post="layer"),
    "d2056": dict(n=11, d=2056, post="rms", groups=11),
    "d4096": dict(n=13, d=4096, pre="rms", post="rms", bias=False, stream="f32"),
    "d4104_f32": dict(n=6, d=4104, dtype="f32", post="layer", groups=2),
    "d8192": dict(n=5, d=8192, post="layer", dh="bf16"),
    "d8200": dict(n=4, d=8200, post="layer", drop=0.5, groups=2),
    "d16384_f32": dict(n=3, d=16384, dtype="f32", post="layer"),
    # what may be absent
    "no_block": dict(n=33, d=384, block=False, gate=False),
    "no_block_rms_f32": dict(n=33, d=200, dtype="f32", block=False, pre="rms"),
    "no_pre": dict(n=21, d=256, pre="none", post="layer"),
    "no_pre_no_post": dict(n=21, d=256, pre="none", gate=True, dtype="f32"),
    "plain_add": dict(n=21, d=256, pre="none", gate=False, bias=False, drop=0.3),
    "no_weights": dict(n=29, d=320, weights=False, bias=False, post="rms"),
    "bias_alone": dict(n=29, d=320, weights=False, post="layer"),
    "no_gate": dict(n=50, d=640, gate=False, post="layer"),
    "no_upstream": dict(n=31, d=128, up=False, post="layer"),
    # groups: a gate for every token, more groups than slices, many rows a group
    "gate_a_token": dict(n=100, d=64, groups=100, post="layer"),
    "groups_70": dict(n=70 * 3, d=128, groups=70, post="layer", drop=0.3),
    "groups_3_long": dict(n=3 * 700, d=72, groups=3, post="layer", dtype="f32"),
    "many_rows": dict(n=2500, d=64, dtype="f32", post="layer", drop=0.1),
    "all_dropped": dict(n=12, d=96, drop=0.999999, post="layer"),
    "empty": dict(n=0, d=128, post="layer"),
    "empty_groups": dict(n=0, d=128, groups=20),
    # a mean far above the deviation: variance taken about the mean
    "offset": dict(n=24, d=768, dtype="f32", offset=300.0, post="layer"),
}


def make(name):
    return Case(**CASES[name], seed=sum(map(ord, name)))


@pytest.mark.parametrize("name", CASES)
def test_forward(name):
    c = make(name)
    say("block norm forward", name, c.n, c.d)
    got = run_forward(c, spoil_dropped=c.row is not None)
    ref = c.forward(c.x, c.y, c.params())
    assert set(got) == set(ref)
    # magnitudes that meet in x_out and h; a deviation's relative error grows
    # with mean over deviation (the rounded subtraction)
    wide = 1.0
    if c.n:
        v = ref["x_out"] if c.block else c.x
        wide = float((v.abs().amax(1) / v.std(1, correction=0).clamp(min=1e-3)).amax()) if c.d > 1 else 1
    yscale = torch.zeros(1, dtype=torch.float64)
    if c.block:
        y = c.y.abs()
        if c.post != "none":
            st = ref["post_stats"]
            n = (c.y - st[:, :1]) * st[:, 1:]
            y = n.abs() + (c.y.abs() + st[:, :1].abs()) * st[:, 1:]
            y = y * (1 if c.post_w is None else c.post_w.abs()) + \
                (0 if c.post_b is None else c.post_b.abs())
        if c.gate is not None:
            y = y * c.gate.abs().repeat_interleave(max(c.n // c.groups, 1), 0)[:c.n]
        yscale = y * abs(c.branch) * (1 if c.row is None else c.row[:, None])
        bound = K * U * (c.x.abs() * abs(c.residual) + yscale)
        close("x_out", got["x_out"], ref["x_out"], bound + rounding(c.stream, ref["x_out"]))
        if c.post != "none":
            mag = c.y.abs().mean(1, keepdim=True) if c.n else c.y[:, :1]
            far = (c.y.abs().amax(1) * ref["post_stats"][:, 1]).clamp(min=1)[:, None] if c.n else mag
            close("post_stats", got["post_stats"], ref["post_stats"],
                  K * U * torch.cat([mag, ref["post_stats"][:, 1:] * far], 1))
    if c.pre != "none":
        st = ref["pre_stats"]
        v = ref["x_out"] if c.block else c.x
        size = c.x.abs() * abs(c.residual) + yscale if c.block else c.x.abs()
        mag = size.mean(1, keepdim=True) if c.n else size[:, :1]
        close("pre_stats", got["pre_stats"], st,
              K * U * torch.cat([mag, st[:, 1:] * max(wide, 1.0)], 1))
        n = (v - st[:, :1]) * st[:, 1:]
        hb = (size + st[:, :1].abs()) * st[:, 1:] + n.abs() * max(wide, 1.0)
        hb = hb * (1 if c.pre_w is None else c.pre_w.abs()) + \
            (0 if c.pre_b is None else c.pre_b.abs())
        close("h", got["h"], ref["h"], K * U * hb + rounding(c.dtype, ref["h"]))


def reference_backward(c, x_out, pre_stats, post_stats):
    """Gradients in float64 from the formulas, and the magnitudes that meet in
    each of them."""
    g, m = {}, {}
    one = torch.ones(c.d, dtype=torch.float64)
    G = c.dx_out.clone() if c.dx_out is not None else torch.zeros(c.n, c.d, dtype=torch.float64)
    GM = G.abs()

    def norm_back(dn, dm, v, stats, kind):
        mu, r = stats[:, :1], stats[:, 1:]
        n = (v - mu) * r
        nm = (v.abs() + mu.abs()) * r
        avg = dn.mean(1, keepdim=True) if kind == "layer" else 0.0
        out = r * (dn - avg - n * (dn * n).mean(1, keepdim=True))
        mag = r * (dm + (dm.mean(1, keepdim=True) if kind == "layer" else 0.0)
                   + nm * (dm * nm).mean(1, keepdim=True))
        return n, nm, out, mag

    if c.pre != "none":
        w = one if c.pre_w is None else c.pre_w
        n, nm, b, bm = norm_back(c.dh * w, (c.dh * w).abs(), x_out, pre_stats, c.pre)
        g["dpre_w"], m["dpre_w"] = (c.dh * n).sum(0), (c.dh.abs() * nm).sum(0)
        g["dpre_b"], m["dpre_b"] = c.dh.sum(0), c.dh.abs().sum(0)
        G, GM = G + b, GM + bm
    scale = c.residual if c.block else 1.0
    g["dx"], m["dx"] = scale * G, abs(scale) * GM
    if c.block:
        a = float(np.float32(c.branch)) * (torch.ones(c.n, dtype=torch.float64) if c.row is None
                                           else c.row)[:, None]
        aG, aM = a * G, a.abs() * GM
        on = a != 0
        gate = torch.ones(1, c.d, dtype=torch.float64) if c.gate is None else c.gate
        gt = gate.repeat_interleave(max(c.n // gate.shape[0], 1), 0)[:c.n]
        w = one if c.post_w is None else c.post_w
        if c.post != "none":
            st = torch.where(on, post_stats, torch.tensor([0.0, 1.0], dtype=torch.float64))
            n, nm, dy, dym = norm_back(aG * gt * w, aM * gt.abs() * w.abs(), c.y, st, c.post)
        else:
            n, nm, dy, dym = c.y, c.y.abs(), aG * gt, aM * gt.abs()
        g["dy"], m["dy"] = torch.where(on, dy, 0.0), dym
        b = 0 if c.post_b is None else c.post_b
        parts = lambda v: v.view(c.groups, -1, c.d).sum(1) if c.n else \
            torch.zeros(c.groups, c.d, dtype=torch.float64)  # noqa: E731
        g["dgate"] = parts(aG * (n * w + b))
        m["dgate"] = parts(aM * (nm * w.abs() + (b.abs() if c.post_b is not None else 0)))
        g["dpost_w"], m["dpost_w"] = (aG * gt * n).sum(0), (aM * gt.abs() * nm).sum(0)
        g["dpost_b"], m["dpost_b"] = (aG * gt).sum(0), (aM * gt.abs()).sum(0)
    return g, m


def saved(c):
    """x_out as the forward stores it and the statistics of the float64 forward
    as f32 holds them."""
    ref = c.forward(c.x, c.y, c.params())
    x_out = ref["x_out"].to(TORCH[c.stream]).double() if c.block else c.x
    f32 = lambda k: ref[k].float().double() if k in ref else None  # noqa: E731
    return x_out, f32("pre_stats"), f32("post_stats")


@pytest.mark.parametrize("name", CASES)
def test_backward(name):
    c = make(name)
    say("block norm backward", name, c.n, c.d)
    at = saved(c)
    got = run_backward(c, *at, spoil_dropped=c.row is not None)
    ref, mag = reference_backward(c, *at)
    types = dict(dx=c.stream, dy=c.dtype)
    for k, t in got.items():
        close(k, t, ref[k], K * U * mag[k] + rounding(types.get(k, "f32"), ref[k]))
    if c.row is not None:
        assert (got["dy"][c.row.cuda() == 0] == 0).all()


@pytest.mark.parametrize("name", ["d192_f32", "groups_3_long", "d2048_f32", "no_pre_no_post",
                                  "no_block_rms_f32", "offset"])
def test_backward_is_the_forwards_gradient(name):
    """Against autograd through the float64 forward, and its directional
    derivative by central differences. The kernel is given what a forward saves,
    so the two differ by the rounding of those to f32."""
    c = make(name)
    leaves = {"x": c.x, "y": c.y, **c.params()}
    leaves = {k: v.clone().requires_grad_() for k, v in leaves.items() if v is not None}

    def objective(v):
        p = {k: v.get(k) for k in c.params()}
        o = c.forward(v["x"], v.get("y"), p)
        s = (o["h"] * c.dh).sum() if "h" in o else 0.0
        return s + ((o["x_out"] * c.dx_out).sum() if c.block else (v["x"] * c.dx_out).sum())

    objective(leaves).backward()
    at = saved(c)
    got = run_backward(c, *at)
    _, mag = reference_backward(c, *at)
    names = dict(x="dx", y="dy", gate="dgate", pre_w="dpre_w", pre_b="dpre_b", post_w="dpost_w",
                 post_b="dpost_b")
    rng = np.random.default_rng(5)
    total, along = 0.0, {}
    for k, v in leaves.items():
        # x_out rounded to f32 and the statistics move n by a few U of what it is made of
        close(names[k], got[names[k]], v.grad, (K + 8 * K) * U * mag[names[k]] + 1e-12)
        along[k] = torch.from_numpy(rng.standard_normal(tuple(v.shape)))
        total += float((got[names[k]].double().cpu() * along[k]).sum())
    e = 1e-5
    with torch.no_grad():
        up = objective({k: v + e * along[k] for k, v in leaves.items()})
        down = objective({k: v - e * along[k] for k, v in leaves.items()})
    slope = float((up - down) / (2 * e))
    size = sum(float((mag[names[k]] * along[k].abs()).sum()) for k in leaves)
    # differences: third derivatives by e^2, and the objective's own 2^-53 over e
    assert abs(total - slope) <= 9 * K * U * size + 1e-6 * size


@pytest.mark.parametrize("name", ["d1000_stream", "d4096", "groups_70", "no_block"])
def test_buffers_shared_and_repeated(name):
    """x_out over x, dx over dx_out and dy over y; the same bits each time."""
    c = make(name)
    a, b = run_forward(c), run_forward(c, in_place=True)
    assert all(same_bits(a[k], b[k]) for k in a)
    at = saved(c)
    a, b = run_backward(c, *at), run_backward(c, *at, in_place=True)
    assert all(same_bits(a[k], b[k]) for k in a)


def test_gradients_left_out():
    c = make("d1000_stream")
    at = saved(c)
    full = run_backward(c, *at)
    for skip in (("dgate",), ("dpost_w", "dpost_b"), ("dpre_w",), ("dpre_b", "dgate"),
                 ("dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")):
        part = run_backward(c, *at, skip=skip)
        assert set(part) == set(full) - set(skip)
        assert all(same_bits(part[k], full[k]) for k in part)


def test_rows_without_variance():
    """A constant row: the layer norm's deviation is sqrt(eps), h is the bias but
    for the mean's rounding."""
    c = make("d192_f32")
    c.pre, c.post = "layer", "none"
    c.pre_b = c.pre_w * 0.5
    c.post_w = None
    c.x[3] = 7.0
    c.y[3] = 0.0
    got = run_forward(c)
    close("h", got["h"][3], c.pre_b, K * U * (7 * EPS ** -0.5 * c.pre_w.abs() + c.pre_b.abs()))
    close("rstd", got["pre_stats"][3, 1:], torch.full((1,), EPS ** -0.5, dtype=torch.float64),
          torch.full((1,), K * U * EPS ** -0.5))


def test_infinities_and_nan_stay_in_their_row():
    c = make("many_rows")
    c.row = None
    clean = run_forward(c)
    c.x[100, 5] = float("inf")
    c.y[200, 7] = float("nan")
    got = run_forward(c)
    rest = torch.ones(c.n, dtype=torch.bool)
    rest[[100, 200]] = False
    for k in ("x_out", "h", "pre_stats"):
        assert same_bits(got[k][rest.cuda()], clean[k][rest.cuda()])
        assert not torch.isfinite(got[k][~rest.cuda()]).all()


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows are those of a call of their own."""
    d, n = 8192, 2 ** 18 + 3
    tail = 5
    say("block norm", n, "x", d, "bf16")
    g = torch.Generator(device="cuda").manual_seed(3)
    bf = torch.bfloat16
    # rows repeat with a period that does not divide the row count
    part = torch.randn(4099, d, device="cuda", generator=g).to(bf)
    x = part.repeat(n // 4099 + 1, 1)[:n]
    y = x.flip(0)
    w = torch.ones(d, dtype=bf, device="cuda")
    s = T.make_norm_shape(n, d, V.VMOE_BF16, dh_dtype=V.VMOE_BF16)
    x_out, h = torch.empty_like(x), torch.empty_like(x)
    st = torch.empty(n, 2, device="cuda")
    T.vmoe_block_norm_fwd(s, x, y, None, None, None, None, w, None, x_out, h, None, st)
    s2 = T.make_norm_shape(tail, d, V.VMOE_BF16, dh_dtype=V.VMOE_BF16)
    xo2, h2, st2 = torch.empty_like(x[:tail]), torch.empty_like(x[:tail]), torch.empty_like(st[:tail])
    T.vmoe_block_norm_fwd(s2, x[-tail:].clone(), y[-tail:].clone(), None, None, None, None, w, None,
                          xo2, h2, None, st2)
    assert same_bits(x_out[-tail:], xo2) and same_bits(h[-tail:], h2) and same_bits(st[-tail:], st2)
    dx, dy = x, y  # their rows are read before they are written
    dw = torch.empty(d, device="cuda")
    ws = torch.empty(T.vmoe_block_norm_bwd_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    last = (x[-tail:].clone(), y[-tail:].clone())
    T.vmoe_block_norm_bwd(s, x, h, x_out, y, None, None, None, None, w, None, st, dx, dy, None, None,
                          None, dw, None, ws)
    dx2, dy2 = torch.empty_like(xo2), torch.empty_like(xo2)
    ws2 = torch.empty(T.vmoe_block_norm_bwd_workspace_bytes(s2), dtype=torch.uint8, device="cuda")
    T.vmoe_block_norm_bwd(s2, last[0], h2, xo2, last[1], None, None, None, None, w, None, st2, dx2,
                          dy2, None, None, None, torch.empty_like(dw), None, ws2)
    assert same_bits(dx[-tail:], dx2) and same_bits(dy[-tail:], dy2)
    assert torch.isfinite(dw).all()


def test_another_stream_and_graph():
    """On a stream of the caller's, and captured once and replayed on new inputs."""
    c = make("d1000_stream")
    ref = run_forward(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run_forward(c, stream=side)
    assert all(same_bits(ref[k], got[k]) for k in ref)

    x, y = _dev(c.x, c.stream), _dev(c.y, c.dtype)
    p = {k: _dev(v, c.dtype) for k, v in c.params().items()}
    row = _dev(c.row, "f32")
    o = dict(x_out=_new(c.n, c.d, c.stream), h=_new(c.n, c.d, c.dtype),
             post_stats=_new(c.n, 2, "f32"), pre_stats=_new(c.n, 2, "f32"))
    s = c.shape()
    ws = torch.empty(T.vmoe_block_norm_bwd_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    dh, up = _dev(c.dh, c.dh_t), _dev(c.dx_out, c.stream)
    b = dict(dx=_new(c.n, c.d, c.stream), dy=_new(c.n, c.d, c.dtype), dpost_w=_new(1, c.d, "f32"),
             dpost_b=_new(1, c.d, "f32"), dgate=_new(1, c.d, "f32"), dpre_w=_new(1, c.d, "f32"),
             dpre_b=_new(1, c.d, "f32"))

    def both():
        T.vmoe_block_norm_fwd(s, x, y, p["post_w"], p["post_b"], p["gate"], row, p["pre_w"],
                              p["pre_b"], o["x_out"], o["h"], o["post_stats"], o["pre_stats"])
        T.vmoe_block_norm_bwd(s, up, dh, o["x_out"], y, p["post_w"], p["post_b"], p["gate"], row,
                              p["pre_w"], o["post_stats"], o["pre_stats"], b["dx"], b["dy"],
                              b["dpost_w"], b["dpost_b"], b["dgate"], b["dpre_w"], b["dpre_b"], ws)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        x.copy_(torch.randn(c.n, c.d, device="cuda") * (k + 1))
        both()
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in {**o, **b}.items()}
        for t in list(o.values()) + list(b.values()) + [ws]:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(t, {**o, **b}[n]) for n, t in eager.items()), k
