"""Launches of vmoe_head.h's calls at the largest sizes that they accept, on the host
alone (the stand-in of test_launch_sizes): each has fewer than 2^32 threads."""
import pytest

from .test_launch_sizes import launches  # noqa: F401

HEAD = """
class Head(ctypes.Structure):
    _fields_ = [(k, I) for k in "n d v k dtype reduction".split()] + \\
        [("temperature", F), ("reserved", I)]
s = Head(*{sizes}, 0, 2.0, 0)
teacher = FAKE if s.k else None
status = lib.vmoe_head_loss_{call}
"""
FWD = "fwd(ctypes.byref(s), *[FAKE] * 4, teacher, teacher, *[FAKE] * 5, MOST, None)"
BWD = "bwd(ctypes.byref(s), FAKE, FAKE, F(1), F(1), *[FAKE] * 4, MOST, None)"

# n, d, v, k, dtype (0: f32, 1: bf16)
LARGEST = [
    (2 ** 21, 8, 2 ** 15 - 1, 256, 1), (2 ** 20, 8, 2 ** 16 - 1, 256, 0),
    (2 ** 21, 504, 1, 256, 1), (2 ** 20, 504, 1, 0, 0),
    (2 ** 15 - 1, 8, 2 ** 21, 256, 1), (2 ** 15 - 1, 8, 2 ** 21, 0, 0),
    (16383, 65536, 2 ** 21, 256, 1), (8191, 65536, 2 ** 21, 256, 0),
    (64, 65536, 2 ** 21, 256, 1), (64, 65536, 2 ** 21, 0, 0), (65, 65536, 2 ** 21, 256, 1),
]


@pytest.mark.parametrize("call", [FWD, BWD], ids=["fwd", "bwd"])
@pytest.mark.parametrize("sizes", LARGEST)
def test_grids_at_the_largest_sizes(launches, call, sizes):  # noqa: F811
    status, noted = launches(HEAD.format(sizes=sizes, call=call))
    assert status == 0 and noted
    for blocks, threads in noted:
        assert 0 < blocks * threads < 2 ** 32 and threads <= 1024


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_rows(launches, dtype):  # noqa: F811
    """Without rows the forward still writes its losses, the backward its dweight."""
    for call in (FWD, BWD):
        status, noted = launches(HEAD.format(sizes=(0, 64, 100, 3, dtype), call=call))
        assert status == 0 and noted
        assert all(blocks > 0 for blocks, _ in noted)
