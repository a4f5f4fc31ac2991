"""What the binding of vmoe_train.h refuses in arguments that are no tensors (no GPU)."""
import pytest
import torch

from paper_2608_16188_amd import vmoe_train as T

from .other_gpu import Elsewhere


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


def test_a_plan_of_two_gpus_refused():
    a, b = Elsewhere(0, 64), Elsewhere(1, 64)
    for bad in ((a, b, a, a), (a, a, a, b)):
        with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
            T.AdamWPlan([T.AdamWTensor(*bad)], device="cpu")
    with pytest.raises(ValueError, match="^param: .*cuda:0.*cuda:1"):
        T.AdamWPlan([T.AdamWTensor(a, a, a, a), T.AdamWTensor(b, b, b, b)], device="cpu")


def test_a_plan_away_from_its_tensors_refused():
    a = Elsewhere(1, 0)
    with pytest.raises(ValueError, match="^device: .*cuda:1.*cpu"):
        T.AdamWPlan([T.AdamWTensor(a, a, a, a)], device="cpu")


def test_a_flag_that_has_no_truth_value_says_so():
    class Odd:
        def __bool__(self):
            raise KeyError("no truth value")

    z = torch.zeros(128, dtype=torch.uint8)
    with pytest.raises(KeyError, match="no truth value"):
        T.vmoe_adamw_state_values(z, z, Odd(), torch.zeros(128))
