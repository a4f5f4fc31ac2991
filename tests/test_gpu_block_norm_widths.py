"""Block norm at widths on the edges and in the middle of every choice of lanes
and waves a row, with the cases, references and bounds of the norm's own tests."""
import pytest
import torch

from . import test_gpu_block_norm as B

pytestmark = pytest.mark.gpu

WIDTHS = {
    "d16_f32": dict(n=150, d=16, dtype="f32", post="layer"),
    "d128": dict(n=70, d=128, post="layer", drop=0.2),
    "d136": dict(n=70, d=136, post="rms", dh="bf16"),
    "d256_groups": dict(n=66, d=256, groups=3, stream="f32", post="layer"),
    "d264": dict(n=35, d=264, post="layer"),
    "d2040": dict(n=17, d=2040, post="layer", groups=17),
    "d3080": dict(n=15, d=3080, post="layer", drop=0.3),
    "d3080_f32": dict(n=10, d=3080, dtype="f32", pre="rms", post="rms", groups=2),
    "d6152": dict(n=7, d=6152, stream="f32", post="layer"),
    "d12296": dict(n=5, d=12296, post="rms", dh="bf16"),
}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", WIDTHS)
def test_widths(name, monkeypatch):
    monkeypatch.setitem(B.CASES, name, WIDTHS[name])
    B.test_forward(name)
    B.test_backward(name)
