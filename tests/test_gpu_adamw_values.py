"""Values of an 8-bit state of more elements than one launch takes."""
import pytest
import torch

from paper_2608_16188_amd import vmoe_train as T

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
    torch.cuda.empty_cache()


def test_more_than_2_32_values():
    """Around the end of a launch and at the end of the state, as those of a small one."""
    n, u8 = 2 ** 32 + 5 * 4096 + 77, torch.uint8
    say("adamw values,", n)
    codes = torch.empty(n, dtype=u8, device="cuda").fill_(0x51)
    scale = torch.empty(-(-n // 128), dtype=u8, device="cuda").fill_(120)
    for a in (2 ** 32 - 8192, n - 4173):
        codes[a:].copy_(torch.randint(0, 256, (n - a,), device="cuda", dtype=u8))
        scale[a // 128:].copy_(torch.randint(90, 150, (scale.numel() - a // 128,), device="cuda",
                                             dtype=u8))
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for signed in (True, False):
        out.fill_(9)
        T.vmoe_adamw_state_values(codes, scale, signed, out)
        for a in (0, 2 ** 32 - 8192):
            b = min(a + 40000, n)
            ref = torch.empty(b - a, dtype=torch.bfloat16, device="cuda")
            T.vmoe_adamw_state_values(codes[a:b].clone(), scale[a // 128:-(-b // 128)].clone(),
                                      signed, ref)
            assert same_bits(out[a:b], ref), (signed, a)
