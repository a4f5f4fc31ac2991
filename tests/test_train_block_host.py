"""What the residual block refuses before it touches the GPU."""
import pytest

from paper_2608_16188_amd import workloads as W
from paper_2608_16188_amd.block import SparseBlock

CFG = W.custom_config("refused", n_tokens=16, d_model=64, d_ff=64, n_experts=2, k=1,
                      capacity_factor=1.0)


@pytest.mark.parametrize("options, match", [
    (dict(norm="none"), "norm: "), (dict(norm="batch"), "norm: "), (dict(norm=None), "norm: "),
    (dict(post_norm="batch"), "post_norm: "), (dict(post_norm=None), "post_norm: "),
    (dict(state_bits=16), "state_bits: "), (dict(state_bits=0), "state_bits: "),
])
def test_options_refused(options, match):
    with pytest.raises(ValueError, match="^" + match):
        SparseBlock(CFG, {}, **options)
