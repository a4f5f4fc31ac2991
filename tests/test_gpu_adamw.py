"""AdamW over many tensors on the GPU: f32 states against float64, 8-bit states
against the format's text in 64-bit integers and floats, rounding statistics,
mixed plans, the gradients' norm and its clip.

Bounds, U = 2^-24: m is two products and a sum, each rounded, of a scaled
gradient (two roundings) and rounded factors: 6 U of the summed magnitudes, v
with its square 9 U. p: the new moments' errors (6 U and half of 9), a square root
and a reciprocal of 1 ulp (2 U) each and some six roundings reach it times lr:
24 U of |update| and 2 U of |p|."""
import math

import numpy as np
import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

from .gpu_common import say
from .train_common import TORCH, U, close, rounding, same_bits

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


# ------------------------------------------------------------------ the text, in numpy

def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_numbers(n, step, seed, index0=0):
    """(r_m, r_v) in (0, 1) for elements index0 .. index0 + n."""
    key = mix(seed ^ mix((step * 0x9E3779B1) & 0xFFFFFFFF))
    i = index0 + np.arange(n, dtype=object) if index0 + n >= 2 ** 32 else \
        index0 + np.arange(n, dtype=np.int64)
    if i.dtype == object:
        bits = np.array([mix(((int(v) & 0xFFFFFFFF) * 0x9E3779B1 & 0xFFFFFFFF)
                             ^ (mix(key ^ (int(v) >> 32)) if int(v) >> 32 else key)) for v in i],
                        dtype=np.int64)
    else:
        bits = mix(((i * 0x9E3779B1) & 0xFFFFFFFF) ^ key)
    return ((bits & 0xFFFF) + 0.5) / 65536, ((bits >> 16) + 0.5) / 65536


def _blocks(x):
    pad = np.zeros(-len(x) % 128, x.dtype)
    return np.concatenate([x, pad]).reshape(-1, 128)


def decode(code, scale, signed):
    """float64 values of codes and scale bytes."""
    bits = 4 if signed else 5
    c = (code & 127 if signed else code).astype(np.int64)
    X, M = c >> 3, c & 7
    top = 2 ** bits - 1
    u = np.where(X > 0, (1 + M / 8) * 2.0 ** (X - top), M / 8 * 2.0 ** (1 - top))
    u = u * 2.0 ** (np.repeat(scale.astype(np.int64), 128)[:len(c)] - 127)
    return np.where(code & 128, -u, u) if signed else u


def encode(x, r, signed):
    """Codes and scale bytes of f32 values x with random numbers r, and which
    codes a last-bit rounding in the linear range may move."""
    bits, low = (4, -14) if signed else (5, -30)
    mag = np.abs(x.astype(np.float32))
    top = _blocks(mag).max(1).view(np.int32).astype(np.int64)
    s = np.minimum((top + 0xFFFFF) >> 23, 255)
    u = mag.astype(np.float64) / 2.0 ** (np.repeat(s, 128)[:len(x)] - 127.0)
    e = np.maximum(np.floor(np.log2(np.where(u > 0, u, 1e-300))), low)
    step = 2.0 ** (e - 3)
    count = np.floor(u / step + r)
    loose = (e == low) & (np.abs(u / step + r - np.round(u / step + r)) < 2.0 ** -19)
    if not signed:
        count = np.where((u > 0) & (count == 0), 1, count)
    code = ((e - low) * 8 + count).astype(np.int64)
    if signed:
        code = code | (np.signbit(x) * 128)
    return code.astype(np.uint8), s.astype(np.uint8), loose


# ------------------------------------------------------------------ one tensor

class One:
    """A tensor with its state on the CPU, as numpy."""

    def __init__(self, n, param="f32", grad="f32", bits=32, seed=0, scale=1e-3, index0=0, lr_mult=1.0,
                 weight_decay=0.1):
        rng = np.random.default_rng(seed)
        self.n, self.ptype, self.gtype, self.bits = n, param, grad, bits
        self.index0, self.lr_mult, self.wd = index0, lr_mult, weight_decay
        self.w = rng.standard_normal(n).astype(np.float32)
        size = scale * np.exp(rng.standard_normal(n))
        self.g = torch.from_numpy((rng.standard_normal(n) * size).astype(np.float32)).to(TORCH[grad])
        if bits == 32:
            self.m = (rng.standard_normal(n) * size).astype(np.float32)
            self.v = (size ** 2 * np.exp(rng.standard_normal(n))).astype(np.float32)
        else:
            b = -(-n // 128)
            self.m = rng.integers(0, 256, n).astype(np.uint8)
            self.v = rng.integers(0, 256, n).astype(np.uint8)
            e = int(round(127 + math.log2(scale)))
            self.ms = rng.integers(e - 3, e + 3, b).astype(np.uint8)
            self.vs = rng.integers(2 * e - 130, 2 * e - 124, b).astype(np.uint8)

    def device(self):
        """AdamWTensor on the GPU; tails of its buffers hold marks."""
        dev = lambda a: torch.from_numpy(np.array(a)).cuda()  # noqa: E731
        master = dev(self.w)
        bf16 = self.ptype == "bf16"
        self.t = T.AdamWTensor(
            param=master.to(torch.bfloat16) if bf16 else master, master=master if bf16 else None,
            grad=self.g.cuda(), m=dev(self.m), v=dev(self.v),
            m_scale=dev(self.ms) if self.bits == 8 else None,
            v_scale=dev(self.vs) if self.bits == 8 else None, lr_mult=self.lr_mult,
            weight_decay=self.wd, index0=self.index0)
        return self.t

    def moments(self):
        if self.bits == 32:
            return self.m.astype(np.float64), self.v.astype(np.float64)
        return decode(self.m, self.ms, True), decode(self.v, self.vs, False)

    def check(self, step, seed=0, grad_scale=1.0, h=HYPER):
        t = self.t
        f = np.float32
        g = self.g.double().numpy() * grad_scale
        m0, v0 = self.moments()
        m = h["beta1"] * m0 + (1 - h["beta1"]) * g
        v = h["beta2"] * v0 + (1 - h["beta2"]) * g * g
        mm = h["beta1"] * np.abs(m0) + (1 - h["beta1"]) * np.abs(g)
        as_t = torch.from_numpy
        up = m / (1 - h["beta1"] ** step) / (np.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"])
        upm = mm / (1 - h["beta1"] ** step) / (np.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"])
        lr = h["lr"] * self.lr_mult
        w = self.w.astype(np.float64)
        p = w - lr * (up + self.wd * w)
        bound = as_t(24 * U * lr * (upm + self.wd * np.abs(w)) + 2 * U * np.abs(w))
        master = t.param if t.master is None else t.master
        close("p", master, as_t(p), bound)
        if t.master is not None:
            assert torch.equal(t.param, t.master.to(torch.bfloat16))
        if self.bits == 32:
            close("m", t.m, as_t(m), as_t(6 * U * mm + 1e-44))
            close("v", t.v, as_t(v), as_t(9 * U * v + 1e-44))
            return
        # moments in f32, each product and sum rounded, as the text has them
        gf = (self.g.float().numpy() * f(grad_scale)).astype(f)
        m32 = m0.astype(f) * f(h["beta1"]) + gf * f(1 - h["beta1"])
        v32 = v0.astype(f) * f(h["beta2"]) + (gf * gf) * f(1 - h["beta2"])
        rm, rv = random_numbers(self.n, step, seed, self.index0)
        for name, got, sc, x, r, signed in (("m", t.m, t.m_scale, m32, rm, True),
                                            ("v", t.v, t.v_scale, v32, rv, False)):
            code, s, loose = encode(x, r, signed)
            assert np.array_equal(sc.cpu().numpy(), s), name
            off = got.cpu().numpy() != code
            assert not (off & ~loose).any(), (name, np.nonzero(off & ~loose)[0][:5])
            assert loose.mean() < 0.01 or self.n < 1000


def step(ones, number, seed=0, clip=None, grad_scale=1.0, stream=None, **h):
    plan = T.AdamWPlan([o.device() for o in ones])
    T.vmoe_adamw(plan, **{**HYPER, **h}, step=number, seed=seed, clip=clip, grad_scale=grad_scale,
                 stream=stream)
    torch.cuda.synchronize()
    return plan


SIZES = [1, 2, 3, 4, 5, 127, 128, 129, 1023, 1024, 1025, 4097, 8191, 8192, 8193, 16384 + 131]
KINDS = [(p, g, b) for p in ("f32", "bf16") for g in ("f32", "bf16") for b in (32, 8)]


@pytest.mark.parametrize("param, grad, bits", KINDS)
def test_sizes(param, grad, bits):
    say("adamw sizes", param, grad, bits)
    # random numbers start at 0, each tensor's after the one before it
    ones = [One(n, param, grad, bits, seed=n, index0=None) for n in SIZES]
    step(ones, 3, seed=77)
    at = 0
    for o in ones:
        o.index0 = at
        o.check(3, seed=77)
        at += -(-o.n // 128) * 128


@pytest.mark.parametrize("param, grad, bits", KINDS)
@pytest.mark.parametrize("n", [1, 129, 8192 + 5])
def test_one_tensor(n, param, grad, bits):
    o = One(n, param, grad, bits, seed=n + bits, index0=640)
    step([o], 1, seed=5)
    o.check(1, seed=5)


def test_mixed_plan():
    """Every kind in one plan, with rates of their own, empty tensors between."""
    ones, at = [], 0
    for i, (p, g, b) in enumerate(KINDS * 3):
        n = SIZES[(5 * i) % len(SIZES)]
        ones.append(One(n, p, g, b, seed=i, index0=at, lr_mult=0.5 * (i % 3), weight_decay=0.2 * (i % 2)))
        at += -(-n // 128) * 128
    empty = T.AdamWTensor(*(torch.empty(0, device="cuda") for _ in range(4)))
    tensors = [o.device() for o in ones]
    plan = T.AdamWPlan(tensors[:7] + [empty] + tensors[7:])
    T.vmoe_adamw(plan, **HYPER, step=12, seed=3)
    torch.cuda.synchronize()
    for o in ones:
        o.check(12, seed=3)


@pytest.mark.parametrize("bits", [32, 8])
def test_views_leave_their_neighbours(bits):
    """Tensors that are parts of flat buffers, of lengths that end inside a
    lane's four elements: what lies between them stays."""
    sizes, gap = [5, 131, 8193, 30], 256
    starts = np.cumsum([0] + [-(-n // 128) * 128 + gap for n in sizes])
    total = int(starts[-1])
    f = lambda dt, v: torch.full((total,), v, dtype=dt, device="cuda")  # noqa: E731
    st = torch.uint8 if bits == 8 else torch.float32
    flat = dict(param=f(torch.bfloat16, 3), master=f(torch.float32, 3), grad=f(torch.bfloat16, 1),
                m=f(st, 9), v=f(st, 9))
    if bits == 8:
        flat.update(m_scale=f(torch.uint8, 120), v_scale=f(torch.uint8, 120))
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    blocks = torch.zeros(total, dtype=torch.bool, device="cuda")
    tensors = []
    for n, a in zip(sizes, starts[:-1]):
        a = int(a)
        inside[a:a + n] = True
        s = slice(a // 128, a // 128 + -(-n // 128))
        blocks[s] = True
        tensors.append(T.AdamWTensor(**{k: t[s] if "scale" in k else t[a:a + n]
                                        for k, t in flat.items()}))
    before = {k: t.clone() for k, t in flat.items()}
    T.vmoe_adamw(T.AdamWPlan(tensors), **HYPER, step=2)
    torch.cuda.synchronize()
    for k, t in flat.items():
        moved = t != before[k]
        assert not (moved & ~(blocks if "scale" in k else inside)).any(), k
    assert (flat["master"][inside] != 3).all()


def test_random_numbers_past_32_bits():
    """index0 around 2^32: the high word changes the numbers."""
    o = One(1024, bits=8, seed=1, index0=2 ** 32 - 512)
    step([o], 4, seed=9)
    o.check(4, seed=9)
    a, b = One(1024, bits=8, seed=2), One(1024, bits=8, seed=2, index0=2 ** 32)
    step([a, b], 4, seed=9)
    assert not torch.equal(a.t.m, b.t.m)


def test_rounding_is_unbiased():
    """Over many seeds the mean of a moment's stored value is its exact one."""
    n, seeds = 256, 4000
    o = One(n, bits=8, seed=11)
    o.device()
    t = o.t
    keep = {k: getattr(t, k).clone() for k in ("param", "m", "v", "m_scale", "v_scale")}
    plan = T.AdamWPlan([t])
    out = torch.empty(n, device="cuda")
    total = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    for seed in range(seeds):
        for k, v in keep.items():
            getattr(t, k).copy_(v)
        T.vmoe_adamw(plan, **HYPER, step=1, seed=seed)
        for i, (c, s) in enumerate(((t.m, t.m_scale), (t.v, t.v_scale))):
            T.vmoe_adamw_state_values(c, s, i == 0, out)
            total[i] += out
    mean = (total / seeds).cpu().numpy()
    m0, v0 = o.moments()
    g = o.g.double().numpy()
    for i, x in enumerate((0.9 * m0 + 0.1 * g, 0.99 * v0 + 0.01 * g * g)):
        top = np.repeat(_blocks(np.abs(x)).max(1), 128)[:n]
        # a step of at most an eighth of the value, or of the linear range's
        unit = np.maximum(np.abs(x) / 8, top * 2.0 ** (-17 if i == 0 else -33) * 2)
        # a mean of `seeds` numbers of deviation at most half a step, 5 sigma, and
        # random numbers in steps of 2^-16
        made_of = 0.9 * np.abs(m0) + 0.1 * np.abs(g) if i == 0 else x
        bound = unit * (0.5 * 5 / math.sqrt(seeds) + 2.0 ** -16) + 9 * U * made_of
        if i == 1:
            bound += top * 2.0 ** -33  # a positive v does not become 0
        assert (np.abs(mean[i] - x) <= bound).all(), i


def test_values_of_states():
    rng = np.random.default_rng(0)
    for n in (1, 3, 128, 300, 8192, 8192 * 2 + 77):
        code = torch.from_numpy(rng.integers(0, 256, n).astype(np.uint8)).cuda()
        scale = torch.from_numpy(rng.integers(60, 200, -(-n // 128)).astype(np.uint8)).cuda()
        for signed in (True, False):
            want = decode(code.cpu().numpy(), scale.cpu().numpy(), signed)
            for dt in (torch.float32, torch.bfloat16):
                out = torch.full((n + 8,), 5.0, dtype=dt, device="cuda")
                T.vmoe_adamw_state_values(code, scale, signed, out[:n])
                torch.cuda.synchronize()
                assert np.array_equal(out[:n].double().cpu().numpy(), want)
                assert (out[n:] == 5).all()


def test_zeros_small_and_large_values():
    """Blocks of zeros, values at both ends of f32's range, single outliers."""
    n = 128 * 6
    o = One(n, bits=8, seed=4)
    g = np.zeros(n, np.float32)
    g[128:256] = 1e-30
    g[256:384] = 1e-42
    g[384:512] = np.linspace(1, 2, 128) * 2.0 ** 60
    g[512:640] = 1e-6
    g[520] = 1.0
    g[640:] = np.float32(2.0 ** -63)
    o.g = torch.from_numpy(g)
    o.m[:], o.v[:], o.ms[:], o.vs[:] = 0, 0, 0, 0
    step([o], 1, seed=8)
    o.check(1, seed=8)
    assert (o.t.m[:128] == 0).all() and (o.t.m_scale[0] == 0).all()
    # v far below its block's largest is kept above 0
    assert (o.t.v[512:640] > 0).all()
    # nothing moves where there never was a gradient, but for the decay
    w = torch.from_numpy(o.w[:128]).double()
    close("decay", o.t.param[:128], w * (1 - 1e-2 * 0.1), 4 * U * w.abs())


def test_not_finite_values_show():
    """An infinity or NaN in a gradient spoils its element, and the state of its
    block in 8 bits, and nothing else."""
    for bits in (32, 8):
        for bad in (float("inf"), float("nan")):
            o, clean = One(1024, bits=bits, seed=6), One(1024, bits=bits, seed=6)
            o.g[300] = bad
            step([o], 2, seed=1)
            step([clean], 2, seed=1)
            rest = torch.ones(1024, dtype=torch.bool)
            rest[300] = False
            assert torch.equal(o.t.param.cpu()[rest], clean.t.param.cpu()[rest])
            assert not torch.isfinite(o.t.param[300])
            rest = torch.ones(1024, dtype=torch.bool)
            rest[256:384] = False
            assert torch.equal(o.t.m.cpu()[rest], clean.t.m.cpu()[rest])
            if bits == 8:
                assert o.t.m_scale[2] == 255 and o.t.v_scale[2] == 255
                out = torch.empty(1024, device="cuda")
                T.vmoe_adamw_state_values(o.t.m, o.t.m_scale, True, out)
                assert not torch.isfinite(out[256:384]).any()


# ------------------------------------------------------------------ norm and clip

def clip_of(ones, max_norm, grad_scale=1.0):
    plan = T.AdamWPlan([o.device() for o in ones])
    clip = torch.full((2,), -1.0, device="cuda")
    ws = torch.full((T.vmoe_grad_norm_workspace_bytes(plan),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    T.vmoe_grad_norm(plan, max_norm, clip, ws, grad_scale)
    return plan, clip


@pytest.mark.parametrize("max_norm, grad_scale", [(math.inf, 1.0), (0.01, 1.0), (1e9, 0.5),
                                                  (0.02, -4.0)])
def test_norm_and_clip(max_norm, grad_scale):
    ones = [One(n, grad=("f32", "bf16")[i % 2], seed=i, index0=0) for i, n in enumerate(SIZES)]
    plan, clip = clip_of(ones, max_norm, grad_scale)
    T.vmoe_adamw(plan, **HYPER, step=5, clip=clip, grad_scale=grad_scale)
    torch.cuda.synchronize()
    norm = abs(grad_scale) * math.sqrt(sum(float(o.g.double().square().sum()) for o in ones))
    got, factor = clip.tolist()
    assert abs(got - norm) <= 64 * U * norm
    want = min(1.0, max_norm / (norm + 1e-6))
    assert abs(factor - want) <= 70 * U * want
    for o in ones:
        o.check(5, grad_scale=grad_scale * factor)


def test_norm_over_many_chunks():
    """More chunks than blocks, and the same bits each time."""
    n = 8192 * 2048 * 2 + 12345
    g = torch.randn(n, device="cuda")
    z = torch.zeros(n, device="cuda")
    plan = T.AdamWPlan([T.AdamWTensor(z, g, z, z)])
    ws = torch.empty(T.vmoe_grad_norm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    a, b = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    T.vmoe_grad_norm(plan, 1.0, a, ws)
    T.vmoe_grad_norm(plan, 1.0, b, ws)
    want = math.sqrt(float(g.double().square().sum()))
    assert same_bits(a, b) and abs(float(a[0]) - want) <= 256 * U * want


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 3e38])
def test_a_norm_that_is_not_finite_skips_the_step(bad):
    ones = [One(n, p, "f32", b, seed=n) for n, p, b in ((500, "f32", 8), (9000, "bf16", 32))]
    ones[1].g[8999] = bad
    plan, clip = clip_of(ones, 1.0)
    before = [{k: v.clone() for k, v in vars(o.t).items() if isinstance(v, torch.Tensor)}
              for o in ones]
    T.vmoe_adamw(plan, **HYPER, step=5, clip=clip)
    torch.cuda.synchronize()
    assert math.isnan(float(clip[1]))
    for o, b in zip(ones, before):
        for k, v in b.items():
            assert same_bits(getattr(o.t, k), v), k


def test_no_tensors():
    plan = T.AdamWPlan([])
    clip = torch.full((2,), -1.0, device="cuda")
    ws = torch.empty(T.vmoe_grad_norm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    T.vmoe_grad_norm(plan, 1.0, clip, ws)
    T.vmoe_adamw(plan, 1e-3, step=1)
    assert clip.tolist() == [0.0, 1.0]


# ------------------------------------------------------------------ over many steps

def test_8bit_states_follow_f32_ones():
    """300 steps on gradients of constant statistics: v (a thousandth a step) keeps
    its size, where rounding to nearest would freeze it, and the weights go the
    way that f32 states take them."""
    n, steps = 65536, 300
    g = torch.Generator(device="cuda").manual_seed(0)
    size = 1e-3 * torch.exp(torch.randn(n // 256, 1, device="cuda", generator=g)).expand(
        -1, 256).reshape(-1)
    mean = 0.5 * size * torch.randn(n, device="cuda", generator=g)
    grad = torch.zeros(n, device="cuda")
    new = lambda bits: T.AdamWTensor(torch.zeros(n, device="cuda"), grad,  # noqa: E731
                                     **T.adamw_state(grad, bits))
    a, b = new(32), new(8)
    plan = T.AdamWPlan([a, b])
    for k in range(steps):
        grad.copy_(mean + size * torch.randn(n, device="cuda", generator=g))
        T.vmoe_adamw(plan, 1e-3, 0.9, 0.999, 1e-8, step=k + 1, seed=42)
    out = torch.empty(n, device="cuda")
    T.vmoe_adamw_state_values(b.v, b.v_scale, False, out)
    ratio = (out / a.v).double()
    assert abs(float(ratio.mean()) - 1) < 0.02 and float(ratio.std()) < 0.35
    rel = float((a.param - b.param).norm() / a.param.norm())
    assert rel < 0.1, rel


def test_streams_and_graph():
    o = One(20000, "bf16", "bf16", 8, seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step([o], 2, seed=4, stream=side)
    o.check(2, seed=4)

    ones = [One(5000, "bf16", "f32", 8, seed=1), One(777, "f32", "bf16", 32, seed=2)]
    plan, clip = clip_of(ones, 0.05)
    ws = torch.empty(T.vmoe_grad_norm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    tensors = [v for o in ones for k, v in vars(o.t).items()
               if isinstance(v, torch.Tensor) and k != "grad"]

    def go():
        T.vmoe_grad_norm(plan, 0.05, clip, ws)
        T.vmoe_adamw(plan, **HYPER, step=3, seed=6, clip=clip)

    start = [t.clone() for t in tensors]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for k in range(3):
        for o in ones:
            o.t.grad.copy_(torch.randn(o.n, device="cuda") * 10.0 ** -k)
        for t, v in zip(tensors, start):
            t.copy_(v)
        go()
        torch.cuda.synchronize()
        eager = [t.clone() for t in tensors]
        for t, v in zip(tensors, start):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(t, e) for t, e in zip(tensors, eager)), k


def test_more_than_2_31_elements():
    """The last elements of a long tensor are those of a small one."""
    n, tail = 2 ** 31 + 8192 + 77, 300
    first = (n - tail) // 128 * 128
    say("adamw", n, "elements")
    u8 = torch.uint8
    grad = torch.empty(n, dtype=torch.bfloat16, device="cuda").fill_(1e-3)
    m = torch.empty(n, dtype=u8, device="cuda").fill_(100)
    v = torch.empty(n, dtype=u8, device="cuda").fill_(200)
    scales = [torch.full((-(-n // 128),), 110, dtype=u8, device="cuda") for _ in range(2)]
    param = torch.empty(n, device="cuda").fill_(0.5)
    grad[first:].copy_(torch.randn(n - first, device="cuda"))
    whole = T.AdamWTensor(param, grad, m, v, m_scale=scales[0], v_scale=scales[1], index0=0)
    part = T.AdamWTensor(*(t[first:].clone() for t in (param, grad, m, v)),
                         m_scale=scales[0][first // 128:].clone(),
                         v_scale=scales[1][first // 128:].clone(), index0=first)
    plan = T.AdamWPlan([whole])
    clip = torch.empty(2, device="cuda")
    ws = torch.empty(T.vmoe_grad_norm_workspace_bytes(plan), dtype=u8, device="cuda")
    T.vmoe_grad_norm(plan, 1e9, clip, ws)
    T.vmoe_adamw(plan, **HYPER, step=2, seed=1)
    T.vmoe_adamw(T.AdamWPlan([part]), **HYPER, step=2, seed=1)
    for k in ("param", "m", "v"):
        assert same_bits(getattr(whole, k)[first:], getattr(part, k)), k
    for k in ("m_scale", "v_scale"):
        assert same_bits(getattr(whole, k)[first // 128:], getattr(part, k)), k
    want = math.sqrt((n - (n - first)) * float(torch.tensor(1e-3).bfloat16()) ** 2
                     + float(grad[first:].double().square().sum()))
    assert abs(float(clip[0]) - want) <= 1e-4 * want
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    T.vmoe_adamw_state_values(whole.m, whole.m_scale, True, out)
    ref = torch.empty(n - first, dtype=torch.bfloat16, device="cuda")
    T.vmoe_adamw_state_values(part.m, part.m_scale, True, ref)
    assert same_bits(out[first:], ref)
