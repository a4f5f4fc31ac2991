"""AdamW's weights where f32 runs out of range: second moments below 2^-126 with
an eps as small, and an eps whose reciprocal is below it.

m and v follow the text operation by operation, so they are given in f32
arithmetic; the weights are the formula in float64 on those. Bound, U = 2^-24: a
square root and a reciprocal of 1 ulp (2 U) each, c1, c2, eps and lr rounded to
f32, and some six operations: 24 U of |update|, 2 U of |p|."""
import numpy as np
import pytest
import torch

from paper_2608_16188_amd import vmoe_train as T

from .gpu_common import say
from .train_common import U, close

pytestmark = pytest.mark.gpu
LR, B1, B2 = 1e-2, 0.9, 0.999


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def check(g, m0, v0, eps, step, bits):
    f = np.float32
    w = np.random.default_rng(1).standard_normal(len(g)).astype(f)
    dev = lambda a: torch.from_numpy(np.array(a)).cuda()  # noqa: E731
    p = dev(w)
    if bits == 32:
        state = dict(m=dev(m0), v=dev(v0))
    else:  # the state is empty: decoded moments are 0
        state = T.adamw_state(p, 8)
        m0, v0 = np.zeros_like(g), np.zeros_like(g)
    T.vmoe_adamw(T.AdamWPlan([T.AdamWTensor(param=p, grad=dev(g), **state)]), LR, B1, B2, eps,
                 step=step)
    torch.cuda.synchronize()
    m = m0 * f(B1) + g * f(1 - B1)
    v = v0 * f(B2) + (g * g) * f(1 - B2)
    if bits == 32:
        assert np.array_equal(state["m"].cpu().numpy(), m)
        assert np.array_equal(state["v"].cpu().numpy(), v)
    c1, c2 = 1 / (1 - B1 ** step), 1 / np.sqrt(1 - B2 ** step)
    up = m.astype(np.float64) * c1 / (np.sqrt(v.astype(np.float64)) * c2 + eps)
    want = w.astype(np.float64) - LR * up
    bound = 24 * U * LR * np.abs(up) + 2 * U * np.abs(w)
    close("p", p, torch.from_numpy(want), torch.from_numpy(bound))
    return up


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-21, 1e-15])
def test_second_moments_below_the_normal_range(eps, bits):
    """Gradients of 1e-23 to 1e-17: v is subnormal for those below 3e-18 and 0
    below some 1e-21."""
    say("adamw subnormal v", eps, bits)
    rng = np.random.default_rng(0)
    n = 1000
    g = (10.0 ** rng.uniform(-23, -17, n) * rng.choice([-1, 1], n)).astype(np.float32)
    g[::50] = 0
    v0 = (10.0 ** rng.uniform(-45, -36, n)).astype(np.float32)
    m0 = (np.sqrt(v0.astype(np.float64)) * rng.standard_normal(n)).astype(np.float32)
    v0[::75] = 0
    check(g, np.zeros_like(g), np.zeros_like(g), eps, 1, bits)
    if bits == 32:
        check(g, m0, v0, eps, 7, bits)


def test_first_step_is_the_learning_rate():
    """Whatever the gradient's size, a first step moves a weight by lr."""
    g = np.full(512, 2e-19, np.float32)
    up = check(g, np.zeros_like(g), np.zeros_like(g), 1e-30, 1, 32)
    assert np.abs(up - 1).max() < 1e-3  # v has some 13 bits


@pytest.mark.parametrize("eps", [2.0 ** 100, 1e38, 3e38])
def test_large_eps(eps):
    """The reciprocal of a denominator above 2^126 is below the normal range."""
    rng = np.random.default_rng(3)
    n = 640
    m0 = (rng.standard_normal(n) * 1e36).astype(np.float32)
    v0 = np.ones(n, np.float32)
    check(rng.standard_normal(n).astype(np.float32), m0, v0, eps, 3, 32)
