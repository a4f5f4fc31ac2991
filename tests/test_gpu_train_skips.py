"""Steps of the residual block whose gradient norm is not finite: nothing
changes and no step is counted."""
import pytest
import torch

from paper_2608_16188_amd import workloads as W
from paper_2608_16188_amd.block import SparseBlock

from .gpu_common import say
from .train_common import same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def make(bits):
    cfg = W.custom_config("skips", n_tokens=96, d_model=64, d_ff=128, n_experts=8, k=2,
                          capacity_factor=0.9, router_std=0.2, noise_var=0.125, dtype=W.BF16)
    return SparseBlock(cfg, W.make_inputs(cfg), gate_init=0.5, state_bits=bits)


def go(b, upstream, stream=None):
    b.forward(stream=stream)
    b.backward(upstream, stream=stream)
    b.update(1e-2, seed=4, stream=stream)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pattern", ["x.", "..x.", ".xx..", "x"])
def test_skipped_steps_do_not_count(pattern, bits):
    """A block with skipped steps (x) is the block that never took them, bit for
    bit: the bias corrections and random numbers go by the steps taken."""
    say("train skips", pattern, bits)
    a, b = make(bits), make(bits)
    gen = torch.Generator(device="cuda").manual_seed(2)
    ups = [torch.randn(96, 64, device="cuda", generator=gen) for _ in pattern]
    side = torch.cuda.Stream()
    for kind, up in zip(pattern, ups):
        if kind == ".":
            go(a, up)
        up = up.clone()
        if kind == "x":
            up[3, 5] = float("nan")
        side.wait_stream(torch.cuda.current_stream())
        go(b, up, side)  # on a stream of the caller's
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert a.steps == b.steps == pattern.count(".")
    for k in a.params:
        assert same_bits(a.params[k], b.params[k]), k
        for s in a.states[k]:
            assert same_bits(a.states[k][s], b.states[k][s]), (k, s)


class Holder:
    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.parametrize("kind", ["stream", "handle", "holder", "default handle"])
def test_streams_as_the_calls_take_them(kind):
    """On a stream that waits: what runs on another one would meet old gradients."""
    a, b = make(32), make(32)
    gen = torch.Generator(device="cuda").manual_seed(5)
    ups = [torch.randn(96, 64, device="cuda", generator=gen) for _ in range(3)]
    for up in ups:
        go(a, up)
    torch.cuda.synchronize()
    side = torch.cuda.default_stream() if kind == "default handle" else torch.cuda.Stream()
    given = {"stream": side, "handle": side.cuda_stream, "holder": Holder(side),
             "default handle": 0}[kind]
    for up in ups:
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
        go(b, up, given)
    side.synchronize()
    assert a.steps == b.steps == 3
    assert all(same_bits(a.params[k], p) for k, p in b.params.items())


def test_steps_can_be_set():
    """As when training goes on from saved parameters and states."""
    a, b = make(32), make(32)
    up = torch.randn(96, 64, device="cuda")
    go(a, up)
    go(b, up)
    b.steps = 40
    assert b.steps == 40
    go(a, up)
    go(b, up)
    assert (a.steps, b.steps) == (2, 41)
    assert not same_bits(a.params["w1"], b.params["w1"])


def test_a_captured_update_is_refused():
    """A replay would repeat the step number that was recorded."""
    b = make(8)
    go(b, torch.randn(96, 64, device="cuda"))
    torch.cuda.synchronize()
    before = {k: p.clone() for k, p in b.params.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward()
        with pytest.raises(RuntimeError, match="captured"):
            b.update(1e-3)
    torch.cuda.synchronize()
    assert b.steps == 1 and all(same_bits(b.params[k], p) for k, p in before.items())
