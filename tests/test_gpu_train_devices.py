"""Tensors of another GPU than the current one are refused before a launch could
reach into it; no second GPU is needed."""
import pytest
import torch

from paper_2608_16188_amd import vmoe as V
from paper_2608_16188_amd import vmoe_train as T

from .other_gpu import Elsewhere

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def test_calls_on_another_gpus_tensors_refused():
    f = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    s = T.make_norm_shape(8, 64, V.VMOE_F32)
    a = dict(x=f(8, 64), y=f(8, 64), post_weight=None, post_bias=None, gate=f(64), row_scale=None,
             pre_weight=f(64), pre_bias=None, x_out=f(8, 64), h=f(8, 64), post_stats=None,
             pre_stats=f(8, 2))
    T.vmoe_block_norm_fwd(s, **a)
    for k in ("x", "gate", "pre_stats"):
        with pytest.raises(ValueError, match="on cuda:[01] is wanted.* got one on cuda:[01]"):
            T.vmoe_block_norm_fwd(s, **{**a, k: Elsewhere(1, *a[k].shape)})
    b = {k: None if t is None else Elsewhere(1, *t.shape) for k, t in a.items()}
    for stream in (None, torch.cuda.Stream()):
        with pytest.raises(ValueError, match="tensors on cuda:1, while the current GPU is cuda:0"):
            T.vmoe_block_norm_fwd(s, **b, stream=stream)
    plan = T.AdamWPlan([T.AdamWTensor(f(64), f(64), f(64), f(64))])
    ws = f(T.vmoe_grad_norm_workspace_bytes(plan), dtype=torch.uint8)
    with pytest.raises(ValueError, match="^clip: .*cuda:"):
        T.vmoe_grad_norm(plan, 1.0, Elsewhere(1, 2), ws)
    with pytest.raises(ValueError, match="cuda:"):
        T.vmoe_grad_norm(plan, 1.0, f(2), Elsewhere(1, 4096, dtype=torch.uint8))
    with pytest.raises(ValueError, match="^clip: .*cuda:"):
        T.vmoe_adamw(plan, 1e-3, clip=Elsewhere(1, 2))
    with pytest.raises(ValueError, match="^out: .*cuda:"):
        T.vmoe_adamw_state_values(f(128, dtype=torch.uint8), f(1, dtype=torch.uint8), True,
                                  Elsewhere(1, 128))
