"""The residual block around the sparse layer: its gradients against float64
autograd through the whole block (routing as the library decided it), and a few
training steps with f32 and 8-bit optimizer states."""
import numpy as np
import pytest
import torch

from paper_2608_16188_amd import workloads as W
from paper_2608_16188_amd.block import SparseBlock, train

from .gpu_common import TOL, say
from .train_common import same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def _config(dtype, groups=1, **kw):
    return W.custom_config("block", n_tokens=groups * 96, d_model=64, d_ff=128, n_experts=8, k=2,
                           capacity_factor=0.9, n_groups=groups, router_std=0.2, noise_var=0.125,
                           dtype=dtype, **kw)


def _reference(b, v, dh, dx_out, eps=1e-6):
    """The block's objective in float64 from the leaves `v`, the library's choices
    and drops held."""
    L, cfg = b.layer, b.layer.cfg
    N, G, E, k = cfg.n_tokens, cfg.n_groups, cfg.n_experts, cfg.k

    def norm(x, w, bias):
        mu = x.mean(1, keepdim=True)
        x = (x - mu) / torch.sqrt((x - mu).square().mean(1, keepdim=True) + eps) * w
        return x + bias

    h = norm(v["x"], v["in_w"], v["in_b"])
    z = torch.matmul(h.view(G, N // G, -1), v["w_router"].transpose(1, 2).contiguous()).view(N, E)
    z = z + L.noise.double().cpu()
    p = torch.softmax(z, 1)
    idx, kept = L.expert_idx.long().cpu(), (L.slot >= 0).double().cpu()
    weight = torch.zeros(N, E, dtype=torch.float64).scatter_add(1, idx, p.gather(1, idx) * kept)
    y = 0
    for e in range(E):
        a = torch.nn.functional.gelu(h @ v["w1"][e].t() + v["b1"][e])
        y = y + weight[:, e:e + 1] * (a @ v["w2"][e].t() + v["b2"][e])
    q = norm(y, v["post_w"], v["post_b"])
    x_out = v["x"] + b.row_scale.double().cpu()[:, None] * v["gate"] * q
    h_out = norm(x_out, v["out_w"], v["out_b"])
    chosen = torch.zeros(N, E, dtype=torch.float64).scatter_add(
        1, idx, torch.ones(N, k, dtype=torch.float64)).view(G, -1, E)
    f = chosen.sum(1) / (k * (N // G))
    balance = E * (f * p.view(G, -1, E).mean(1)).sum()
    z_loss = torch.logsumexp(z, 1).square().view(G, -1).mean(1).sum()
    return (h_out * dh).sum() + (x_out * dx_out).sum() + b.w_balance * balance + b.w_z * z_loss


@pytest.mark.parametrize("groups", [1, 3])
def test_gradients_of_the_whole_block(groups):
    cfg = _config(W.F32, groups)
    say("train block gradients", groups)
    b = SparseBlock(cfg, W.make_inputs(cfg), post_norm="layer", gate_init=0.7, row_scale=True,
                    w_balance=0.5, w_z=0.05)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    for name in ("in_w", "in_b", "post_w", "post_b", "out_w", "out_b", "gate"):
        b.params[name].add_(0.2 * rand(64))
    b.row_scale.copy_((rand(cfg.n_tokens) > -0.8).float() * 1.25)
    dh, up = rand(cfg.n_tokens, 64), rand(cfg.n_tokens, 64)
    b.forward()
    b.backward(dh, up)
    torch.cuda.synchronize()
    leaves = {k: t.detach().double().cpu().requires_grad_() for k, t in
              {**b.params, "x": b.x}.items()}
    _reference(b, leaves, dh.double().cpu(), up.double().cpu()).backward()
    for k, t in {**b.grads, "x": b.dx}.items():
        ref = leaves[k].grad
        err = float((t.double().cpu().view_as(ref) - ref).abs().max() / ref.abs().max())
        assert err <= TOL[W.F32], (k, err)


@pytest.mark.parametrize("dtype", [W.F32, W.BF16])
def test_training_lowers_the_loss(dtype):
    cfg = _config(dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    target = torch.randn(cfg.n_tokens, 64, device="cuda", generator=gen)
    ends = {}
    for bits in (32, 8):
        say("train block", dtype, bits)
        block, losses = train(cfg, W.make_inputs(cfg), target, 120, 1e-2, state_bits=bits,
                              gate_init=0.5)
        assert all(np.isfinite(losses)) and losses[-1] < 0.6 * losses[0], losses[::20]
        ends[bits] = losses[-1]
        assert block.demand.sum() == cfg.n_tokens * cfg.k
    assert abs(ends[8] - ends[32]) < 0.1 * ends[32], ends


def test_a_step_repeats_and_captures():
    """Forward and backward: the same bits again, and from a graph."""
    cfg = _config(W.BF16, 3)
    b = SparseBlock(cfg, W.make_inputs(cfg), norm="rms", post_norm="rms")
    dh = torch.randn(cfg.n_tokens, 64, device="cuda")

    def go():
        b.forward()
        b.backward(dh)

    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    outs = dict(b.grads, x=b.dx, h=b.h_out, losses=b.losses, demand=b.demand)
    for k in range(3):
        b.x.copy_(torch.randn(cfg.n_tokens, 64, device="cuda"))
        go()
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in outs.items()}
        for t in outs.values():
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(outs[n], t) for n, t in eager.items()), k
