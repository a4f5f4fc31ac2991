"""What the binding of vmoe_train.h refuses in arguments that are no tensors (no GPU)."""
import pytest

from paper_2608_16188_amd import vmoe_train as T


def plan():
    p = T.AdamWPlan([], device="cpu")
    assert p.n_chunks == 0  # nothing is launched
    return p


@pytest.mark.parametrize("seed", [-1, 1 << 32, (1 << 32) + 5, -(1 << 40)])
def test_seeds_outside_32_bits_refused(seed):
    with pytest.raises(ValueError, match="seed: "):
        T.vmoe_adamw(plan(), 1e-3, seed=seed, stream=0)


@pytest.mark.parametrize("seed", [0, 5, (1 << 32) - 1])
def test_seeds_of_32_bits_accepted(seed):
    T.vmoe_adamw(plan(), 1e-3, seed=seed, stream=0)
