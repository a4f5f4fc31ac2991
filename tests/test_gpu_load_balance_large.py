"""Load-balance loss on gates of more than 16 MB of probs, which take launches of
their own for the counts, the rows and the losses, and groups without a live
token where a group takes more than one block.

Bounds as for the smaller gates, with a lane's sums ended by its chunk: a lane
adds at most a 32nd of a chunk's tokens in f32, then 10 levels of lanes and
waves; chunks meet in double."""
import pytest
import torch

from .gpu_common import say
from .test_gpu_load_balance import Case, run
from .train_common import U, close, same_bits

pytestmark = pytest.mark.gpu

# name: groups, tokens a group, E, k, bias, noise, padding
CASES = {
    "e64_one_group": (1, 70001, 64, 6, True, True, 0.2),
    "e33_groups": (5, 27011, 33, 3, True, False, 0.1),
    "e13_groups": (17, 20011, 13, 4, False, True, 0.5),
    "e8_one_group": (1, 560003, 8, 2, False, True, 0.0),
    "e3_one_group": (1, 1500001, 3, 1, False, False, 0.3),
    "e64_many_groups": (200, 351, 64, 2, False, False, 0.0),
    "e64_more_groups_than_chunks": (700, 263, 64, 2, True, False, 0.2),
    "e32_a_group_of_padding": (3, 47003, 32, 4, False, True, 0.1),
}
TWO_LAUNCHES = {
    "e32_a_group_of_padding": (3, 2003, 32, 4, False, True, 0.1),
    "e7_groups_of_padding": (4, 5001, 7, 2, True, False, 0.4),
}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def make(name, cases=CASES):
    c = Case(*cases[name], seed=sum(map(ord, name)))
    if "of_padding" in name:  # every other group, the first one live
        c.mask.view(c.G, -1)[1::2] = 0
    return c


def check(c):
    got = run(c)
    losses, demand, mean, grad, mag, zmag = c.reference()
    assert torch.equal(got["demand"].cpu(), demand)
    chunk = -(-(c.n // c.G) // max(512 // c.G, 1))
    adds = chunk / 32 + 32
    close("mean_probs", got["mean_probs"], mean, adds * U * mean)
    close("dlogits", got["dlogits"], grad, 24 * U * mag)
    sq = torch.where(c.live(), zmag ** 2, 0.0).view(c.G, -1).sum(1)
    lz = (adds + 16) * U * sq / c.live().view(c.G, -1).sum(1).clamp(min=1)
    close("losses", got["losses"], losses,
          torch.stack([adds * U * losses[:, 0], lz], 1) + 1e-30)
    if c.mask is not None:
        assert (got["dlogits"][(c.mask == 0).cuda()] == 0).all()
    return got


@pytest.mark.parametrize("name", CASES)
def test_large_gates(name):
    c = make(name)
    say("load balance, large", name, c.n, c.E, c.k)
    assert 4 * c.n * c.E > 16 << 20
    got = check(c)
    again = run(c)
    assert all(same_bits(again[k], got[k]) for k in got)


@pytest.mark.parametrize("name", TWO_LAUNCHES)
def test_groups_without_a_live_token(name):
    c = make(name, TWO_LAUNCHES)
    assert 4 * c.n * c.E <= 16 << 20
    got = check(c)
    for k in ("losses", "demand", "mean_probs"):
        assert (got[k][1::2] == 0).all(), k


def test_more_groups_than_a_launch_has_blocks():
    c = Case((1 << 21) + 5, 1, 2, 1, True, False, 0.3, seed=8)
    say("load balance", c.G, "groups")
    check(c)


def test_a_large_gate_from_a_graph():
    from paper_2608_16188_amd import vmoe_train as T
    c = make("e33_groups")
    s = c.shape()
    logits, probs, idx, bias = c.logits.cuda(), c.probs.cuda(), c.idx.cuda(), c.bias.cuda()
    mask = c.mask.cuda()
    o = dict(losses=torch.empty(c.G, 2, device="cuda"),
             demand=torch.empty(c.G, c.E, dtype=torch.int32, device="cuda"),
             mean_probs=torch.empty(c.G, c.E, device="cuda"),
             dlogits=torch.empty(c.n, c.E, device="cuda"))
    ws = torch.empty(T.vmoe_load_balance_loss_workspace_bytes(s), dtype=torch.uint8, device="cuda")

    def go():
        T.vmoe_load_balance_loss(s, logits, bias, None, probs, idx, mask, 0.01, 0.002, o["losses"],
                                 o["demand"], o["mean_probs"], o["dlogits"], ws)

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
