"""Load-balance loss on the GPU against its definition in float64.

Bounds: demand is exact. mean_probs: sums of non-negative f32, a lane at most
N / 32 of them at the sizes here with one block a group and far fewer with
chunks, 10 levels of lanes and waves, doubles beyond: N/32 + 32 roundings of
U = 2^-24. lse: a rounding of max z and of log max p each, and probs' own error
(the softmax that the test hands over is rounded from float64): 8 U (|max z| +
|log max p| + 1). dlogits: some 10 roundings of its terms' magnitudes and lse's."""
import numpy as np
import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T
from paper_2608_16188_amd import workloads as W
from paper_2608_16188_amd.layer import LayerBuffers

from .gpu_common import say
from .train_common import U, close, same_bits

pytestmark = pytest.mark.gpu
WB, WZ = 0.01, 0.002


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


# name: groups, tokens a group, E, k, bias, noise, padding
CASES = {
    "one_token_one_expert": (1, 1, 1, 1, False, False, 0.0),
    "one_token": (1, 1, 8, 2, True, True, 0.0),
    "two_experts": (1, 33, 2, 1, False, True, 0.0),
    "e3_k3": (2, 50, 3, 3, True, False, 0.3),
    "e5_odd": (3, 257, 5, 2, True, True, 0.1),
    "e8_one_image": (1, 197, 8, 2, False, True, 0.0),
    "e13_groups": (17, 91, 13, 4, False, False, 0.5),
    "e16_edge_of_one_block": (1, 1024, 16, 2, False, True, 0.0),
    "e16_past_one_block": (1, 1025, 16, 2, True, True, 0.2),
    "e4_past_one_block": (1, 2049, 4, 1, False, False, 0.0),
    "e32_hot": (1, 5000, 32, 2, True, True, 0.0),
    "e33": (2, 700, 33, 3, True, False, 0.1),
    "e63_chunks": (3, 1999, 63, 8, False, True, 0.4),
    "e64_k8": (1, 3001, 64, 8, True, True, 0.0),
    "e64_k64": (1, 130, 64, 64, False, False, 0.0),
    "many_groups": (1500, 3, 8, 2, False, False, 0.5),
    "long_e8": (1, 36928, 8, 2, False, True, 0.1),
    "all_padding": (2, 700, 8, 2, False, True, 1.0),
    "empty": (3, 0, 8, 2, False, False, 0.0),
}


class Case:
    def __init__(self, G, Ng, E, k, bias, noise, padding, seed):
        rng = np.random.default_rng(seed)
        n = G * Ng
        self.G, self.E, self.k, self.n = G, E, k, n
        f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32))  # noqa: E731
        self.logits = f32(rng.standard_normal((n, E)) * 1.5)
        self.bias = f32(rng.standard_normal(E)) if bias else None
        self.noise = f32(rng.standard_normal((n, E)) * 0.3) if noise else None
        self.mask = None
        if padding:
            self.mask = torch.from_numpy((rng.random(n) >= padding).astype(np.uint8) * 3)
        z = self.z()
        self.probs = torch.softmax(z, 1).float()
        self.idx = torch.topk(z, k, 1).indices.to(torch.int32)

    def z(self):
        """Noisy logits as f32 holds them, in float64."""
        z = self.logits
        z = z + self.bias if self.bias is not None else z
        return (z + self.noise if self.noise is not None else z).double()

    def live(self):
        return torch.ones(self.n, dtype=torch.bool) if self.mask is None else self.mask != 0

    def shape(self):
        return V.make_shape(self.n, self.G, 64, 64, self.E, self.k, 1.0, V.VMOE_F32)

    def reference(self, wb=WB, wz=WZ):
        """losses, demand, mean_probs, dlogits and the magnitudes of dlogits."""
        G, E, k = self.G, self.E, self.k
        live = self.live()
        p = torch.where(live[:, None], self.probs.double(), 0.0).view(G, -1, E)
        lse = torch.where(live, torch.logsumexp(self.z(), 1), 0.0).view(G, -1)
        one = torch.zeros(self.n, E, dtype=torch.int64).scatter_add_(
            1, self.idx.long(), torch.ones(self.n, k, dtype=torch.int64))
        demand = (one * live[:, None]).view(G, -1, E).sum(1)
        count = live.view(G, -1).sum(1).clamp(min=1).double()[:, None]
        f = demand.double() / (k * count)
        mean = p.sum(1) / count
        losses = torch.stack([E * (f * mean).sum(1), (lse ** 2).sum(1) / count[:, 0]], 1)
        inner = (p * f[:, None]).sum(2, keepdim=True)
        scale = p / count[:, :, None]
        grad = scale * (wb * E * (f[:, None] - inner) + 2 * wz * lse[:, :, None])
        zmag = self.z().abs().amax(1) + torch.log(self.probs.double().amax(1)).abs() + 1 \
            if self.n else torch.zeros(0, dtype=torch.float64)
        mag = scale * (wb * E * (f[:, None] + inner) + 2 * wz * zmag.view(G, -1)[:, :, None])
        return losses, demand.int(), mean, grad.view(self.n, E), mag.view(self.n, E), zmag


def make(name):
    return Case(*CASES[name], seed=sum(map(ord, name)))


def run(c, spoil=True, mean=True, wb=WB, wz=WZ, stream=None):
    """spoil: what padding rows hold is not to matter."""
    def dev(t):
        if t is None:
            return None
        return (t if t.numel() else torch.zeros(16, dtype=t.dtype)).cuda()

    a = dict(logits=dev(c.logits), noise=dev(c.noise), probs=dev(c.probs), idx=dev(c.idx))
    if spoil and c.mask is not None and c.n:
        off = (c.mask == 0).cuda()
        a["logits"][off] = float("nan")
        a["probs"][off] = float("inf")
        if a["noise"] is not None:
            a["noise"][off] = torch.finfo(torch.float32).min
        a["idx"][off] = 2 ** 31 - 1
    s = c.shape()
    o = dict(losses=torch.full((c.G, 2), float("nan"), device="cuda"),
             demand=torch.full((c.G, c.E), -5, dtype=torch.int32, device="cuda"),
             mean_probs=torch.full((c.G, c.E), float("nan"), device="cuda") if mean else None,
             dlogits=torch.full((max(c.n, 1), c.E), float("nan"), device="cuda"))
    ws = torch.full((max(T.vmoe_load_balance_loss_workspace_bytes(s), 16),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    T.vmoe_load_balance_loss(s, a["logits"], dev(c.bias), a["noise"], a["probs"], a["idx"],
                             dev(c.mask), wb, wz, o["losses"], o["demand"], o["mean_probs"],
                             o["dlogits"], ws, stream)
    torch.cuda.synchronize()
    o["dlogits"] = o["dlogits"][:c.n]
    return o


@pytest.mark.parametrize("name", CASES)
def test_against_float64(name):
    c = make(name)
    say("load balance", name, c.n, c.E, c.k)
    got = run(c)
    losses, demand, mean, grad, mag, zmag = c.reference()
    assert torch.equal(got["demand"].cpu(), demand)
    adds = c.n / 32 + 32
    close("mean_probs", got["mean_probs"], mean, adds * U * mean)
    close("dlogits", got["dlogits"], grad, 24 * U * mag)
    lb = adds * U * losses[:, 0]
    lz = torch.zeros(c.G, dtype=torch.float64)
    if c.n:
        sq = torch.where(c.live(), zmag ** 2, 0.0).view(c.G, -1).sum(1)
        lz = (adds + 16) * U * sq / c.live().view(c.G, -1).sum(1).clamp(min=1)
    close("losses", got["losses"], losses, torch.stack([lb, lz], 1) + 1e-30)
    if c.mask is not None:
        assert (got["dlogits"][(c.mask == 0).cuda()] == 0).all()


@pytest.mark.parametrize("name", ["e5_odd", "e13_groups", "e63_chunks", "e32_hot"])
def test_gradient_against_differences(name):
    """Directional derivative of the float64 objective in the logits (demand held:
    it is piecewise constant), softmax and all."""
    c = make(name)
    got = run(c)["dlogits"].double().cpu()
    live = c.live()
    f = (c.reference()[1].double() / (c.k * live.view(c.G, -1).sum(1).clamp(min=1)[:, None]))
    rng = np.random.default_rng(1)
    along = torch.from_numpy(rng.standard_normal((c.n, c.E)))

    def objective(z):
        p = torch.softmax(z, 1) * live[:, None]
        n = live.view(c.G, -1).sum(1).clamp(min=1)
        P = p.view(c.G, -1, c.E).sum(1) / n[:, None]
        lse = torch.logsumexp(z, 1) * live
        return (WB * c.E * (f * P).sum(1) + WZ * (lse ** 2).view(c.G, -1).sum(1) / n).sum()

    e = 1e-5
    slope = (objective(c.z() + e * along) - objective(c.z() - e * along)) / (2 * e)
    mag = c.reference()[4]
    assert abs(float((got * along).sum() - slope)) <= float((mag * along.abs()).sum()) * 1e-5


def test_even_load_and_one_expert():
    """An even gate has a balance loss of 1; one expert that takes all, E."""
    n, E = 640, 8
    c = Case(1, n, E, 1, False, False, 0.0, 3)
    c.logits = torch.zeros(n, E)
    c.probs = torch.full((n, E), 1 / E)
    c.idx = (torch.arange(n) % E).int()[:, None]
    o = run(c)
    close("even", o["losses"][0], torch.tensor([1.0, float(np.log(E)) ** 2]),
          torch.tensor([1e-6, 1e-5]))
    c.probs = torch.zeros(n, E)
    c.probs[:, 3] = 1.0
    c.logits[:, 3] = 200.0
    c.idx = torch.full((n, 1), 3, dtype=torch.int32)
    o = run(c)
    close("one", o["losses"][0], torch.tensor([float(E), 200.0 ** 2]), torch.tensor([1e-5, 0.1]))
    assert o["demand"][0].tolist() == [0, 0, 0, n, 0, 0, 0, 0]


@pytest.mark.parametrize("off", [float("-inf"), torch.finfo(torch.float32).min])
def test_disabled_experts(off):
    """An offset of the lowest value or of -infinity switches an expert off."""
    c = Case(2, 300, 16, 2, True, True, 0.0, 9)
    c.bias[4:7] = off
    z = c.z()
    c.probs = torch.softmax(z, 1).float()
    c.idx = torch.topk(z, 2, 1).indices.int()
    o = run(c)
    losses, demand, mean, grad, _, _ = c.reference()
    assert torch.equal(o["demand"].cpu(), demand) and (o["demand"][:, 4:7] == 0).all()
    assert (o["dlogits"][:, 4:7] == 0).all() and (o["mean_probs"][:, 4:7] == 0).all()
    close("dlogits", o["dlogits"], grad, 1e-5 * grad.abs().amax() + 0 * grad)
    close("losses", o["losses"], losses, 1e-5 * losses)


def test_indices_outside_are_not_counted():
    c = make("e8_one_image")
    c.idx[5] = torch.tensor([-1, 8], dtype=torch.int32)
    c.idx[6] = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    o = run(c)
    want = torch.bincount(c.idx[(c.idx >= 0) & (c.idx < 8)].long(), minlength=8)
    assert torch.equal(o["demand"][0].cpu().long(), want)


@pytest.mark.parametrize("name", ["e8_one_image", "e63_chunks"])
def test_weights_alone_and_optional_output(name):
    c = make(name)
    both = run(c)
    a, b = run(c, wb=WB, wz=0.0), run(c, wb=0.0, wz=WZ, mean=False)
    assert same_bits(a["losses"], both["losses"]) and same_bits(b["losses"], both["losses"])
    mag = c.reference()[4]
    close("sum", a["dlogits"] + b["dlogits"], both["dlogits"].double().cpu(), 16 * U * mag)
    again = run(c)
    assert all(same_bits(again[k], both[k]) for k in both)


def test_stream_and_graph():
    c = make("e63_chunks")
    ref = run(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(c, stream=side)
    assert all(same_bits(got[k], ref[k]) for k in ref)
    s = c.shape()
    logits, probs, idx = c.logits.cuda(), c.probs.cuda(), c.idx.cuda()
    noise, mask = c.noise.cuda(), c.mask.cuda()
    o = dict(losses=torch.empty(c.G, 2, device="cuda"),
             demand=torch.empty(c.G, c.E, dtype=torch.int32, device="cuda"),
             dlogits=torch.empty(c.n, c.E, device="cuda"))
    ws = torch.empty(T.vmoe_load_balance_loss_workspace_bytes(s), dtype=torch.uint8, device="cuda")

    def go():
        T.vmoe_load_balance_loss(s, logits, None, noise, probs, idx, mask, WB, WZ, o["losses"],
                                 o["demand"], None, o["dlogits"], ws)

    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for k in range(3):
        mask.copy_((torch.rand(c.n, device="cuda") < 0.3 * (k + 1)).to(torch.uint8))
        go()
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in o.items()}
        for t in list(o.values()) + [ws]:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(o[n], t) for n, t in eager.items()), k


def test_with_the_layers_routing():
    """Fed by vmoe_route: demand is at least what the experts keep, and the loss
    gradient reaches the router through the layer's backward."""
    cfg = W.custom_config("balance", n_tokens=3 * 130, d_model=64, d_ff=64, n_experts=8, k=2,
                          capacity_factor=0.7, n_groups=3, router_std=0.2, noise_var=0.1)
    L = LayerBuffers(cfg, W.make_inputs(cfg))
    L.forward()
    f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    losses, dl = f(3, 2), f(390, 8)
    demand = torch.empty(3, 8, dtype=torch.int32, device="cuda")
    ws = torch.empty(T.vmoe_load_balance_loss_workspace_bytes(L.shape), dtype=torch.uint8,
                     device="cuda")
    T.vmoe_load_balance_loss(L.shape, L.logits, L.logit_bias, L.noise, L.probs, L.expert_idx, None,
                             WB, WZ, losses, demand, None, dl, ws)
    L.backward()
    plain = L.dx.clone(), L.dw_router.clone()
    L.backward(dlogits=dl)
    torch.cuda.synchronize()
    assert (demand.sum(1) == 260).all() and (demand >= L.counts).all()
    assert torch.equal(torch.minimum(demand, torch.full_like(demand, L.C)), L.counts)
    wr = L.w_router.float().view(3, 8, 64)
    extra = torch.matmul(dl.view(3, 130, 8), wr).view(390, 64)
    assert torch.allclose(L.dx - plain[0], extra, atol=2e-5 * float(L.dx.abs().max()))
    extra = torch.matmul(dl.view(3, 130, 8).transpose(1, 2).contiguous(),
                         L.x.float().view(3, 130, 64))
    assert torch.allclose(L.dw_router - plain[1], extra,
                          atol=2e-5 * float(L.dw_router.abs().max()))
