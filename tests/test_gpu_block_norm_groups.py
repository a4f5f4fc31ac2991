"""Block norm's backward with a gate row for each of millions of tokens, whose
blocks and whose gate's sums take more than one launch: rows and gate gradients
at both ends are those of calls of their own, the weights' gradients float64's."""
import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

from .gpu_common import say
from .train_common import U, close, same_bits

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def backward(x, y, up, dh, gate, stats, w, weights):
    n, d = x.shape
    s = T.make_norm_shape(n, d, V.VMOE_BF16, n_groups=n, dh_dtype=V.VMOE_BF16)
    o = dict(dx=torch.empty_like(x), dy=torch.empty_like(y),
             dgate=torch.empty(n, d, device="cuda"))
    dw, db = (torch.empty(d, device="cuda") if weights else None for _ in range(2))
    ws = torch.empty(T.vmoe_block_norm_bwd_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    T.vmoe_block_norm_bwd(s, up, dh, x, y, None, None, gate, None, w, None, stats, o["dx"],
                          o["dy"], None, None, o["dgate"], dw, db, ws)
    torch.cuda.synchronize()
    return o, dw, db


# 2^23 blocks of 256 threads a launch; 2^21 blocks of 1024 for the gates' sums
@pytest.mark.parametrize("n, d", [((1 << 23) + 37, 8), ((1 << 22) + 70, 512)])
def test_a_gate_for_each_token(n, d):
    say("block norm backward,", n, "groups x", d)
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda: torch.randn(n, d, device="cuda", dtype=BF, generator=g)  # noqa: E731
    x, y, up, dh, gate = (rand() for _ in range(5))
    w = (1 + 0.1 * torch.randn(d, device="cuda", generator=g)).to(BF)
    stats = torch.rand(n, 2, device="cuda", generator=g) + 0.5
    weights = d == 8
    o, dw, db = backward(x, y, up, dh, gate, stats, w, weights)
    for part in (slice(0, 50), slice(n // 2, n // 2 + 50), slice(n - 50, n)):
        p, _, _ = backward(*(t[part].clone() for t in (x, y, up, dh, gate, stats)), w, False)
        for k in o:
            assert same_bits(o[k][part], p[k]), k
    if weights:
        # a column's slice adds a 32nd of the rows in f32, then the slices
        unit = (x.double() - stats[:, :1]) * stats[:, 1:]
        far = (x.double().abs() + stats[:, :1]) * stats[:, 1:]
        adds = n / 32 + 64
        close("dpre_w", dw, (dh.double() * unit).sum(0),
              adds * U * (dh.double().abs() * far).sum(0))
        close("dpre_b", db, dh.double().sum(0), adds * U * dh.double().abs().sum(0))
