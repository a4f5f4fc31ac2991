"""Launches of vmoe_train.h's calls at the largest sizes that they accept, on the
host alone: a small library stands in for the runtime's launch calls and notes
each grid. A launch has to have fewer than 2^32 threads."""
import json
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2608_16188_amd import vmoe as V

STUB = r"""
typedef struct { unsigned x, y, z; } dim3_t;
static dim3_t grid, block;
static unsigned long noted[4096][2];
static int n;
int __hipPushCallConfiguration(dim3_t g, dim3_t b, unsigned long shared, void* stream) {
    grid = g;
    block = b;
    (void)shared, (void)stream;
    return 0;
}
int __hipPopCallConfiguration(dim3_t* g, dim3_t* b, unsigned long* shared, void** stream) {
    *g = grid;
    *b = block;
    *shared = 0;
    *stream = 0;
    return 0;
}
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, unsigned long shared,
                    void* stream) {
    (void)f, (void)args, (void)shared, (void)stream;
    if (n < 4096) {
        noted[n][0] = (unsigned long)g.x * g.y * g.z;
        noted[n][1] = (unsigned long)b.x * b.y * b.z;
    }
    ++n;
    return 0;
}
int hipGetLastError(void) { return 0; }
int count(void) { return n; }
unsigned long blocks(int i) { return noted[i][0]; }
unsigned long threads(int i) { return noted[i][1]; }
"""

# No torch here: the stand-in has to be found before the runtime itself.
CALLER = r"""
import ctypes, json, sys
stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
stub.blocks.restype = stub.threads.restype = ctypes.c_ulong
P, I, L, F, D = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double)
FAKE = P(0x10000)
MOST = ctypes.c_size_t(1 << 62)
class Norm(ctypes.Structure):
    _fields_ = [(k, I) for k in "n g d dtype stream dh pre post".split()] + \
        [(k, F) for k in "eps residual branch".split()] + [("reserved", I)]
class Shape(ctypes.Structure):
    _fields_ = [(k, I) for k in "n g d f e k".split()] + [("factor", D)] + \
        [(k, I) for k in "rounding override dtype reserved".split()]
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """A function: the caller's lines -> (status, [(blocks, threads a block)])."""
    folder = tmp_path_factory.mktemp("launches")
    src, lib = folder / "stub.c", folder / "libstub.so"
    src.write_text(STUB)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", str(src), "-o", str(lib)])

    def run(text):
        code = CALLER + textwrap.dedent(text) + textwrap.dedent("""
            print(json.dumps([status, [(stub.blocks(i), stub.threads(i))
                                       for i in range(stub.count())]]))""")
        out = subprocess.run([sys.executable, "-c", code, str(lib), V.LIB_PATH], check=True,
                             capture_output=True, text=True, cwd=os.path.dirname(__file__)).stdout
        status, noted = json.loads(out.splitlines()[-1])
        assert len(noted) < 4096
        return status, noted

    return run


def fits(noted):
    assert noted and all(0 < b * t < 1 << 32 for b, t in noted), noted


LOSS = """
    s = Shape({n}, {g}, 8, 8, {e}, {k}, 1.0, 0, 0, 0, 0)
    status = lib.vmoe_load_balance_loss(ctypes.byref(s), *[FAKE] * 6, F(1), F(1), *[FAKE] * 4, FAKE,
                                        MOST, None)
"""


@pytest.mark.parametrize("n, g, e, k", [
    (1 << 21, 1 << 21, 64, 1), (1 << 22, 1 << 22, 8, 2), ((1 << 22) + 5, (1 << 22) + 5, 8, 1),
    ((1 << 25) - 1, (1 << 25) - 1, 8, 1), (3 << 24, 1 << 24, 2, 1),
    ((1 << 26) - 1, (1 << 26) - 1, 1, 1)])
def test_groups_of_the_loss_each_in_a_block(launches, n, g, e, k):
    status, noted = launches(LOSS.format(n=n, g=g, e=e, k=k))
    assert status == V.VMOE_OK
    fits(noted)
    assert sum(b for b, _ in noted) == g


@pytest.mark.parametrize("n, g, e, k", [
    (1 << 24, 1, 64, 1), (130000 * 257, 130000, 64, 1), ((1 << 26) - 1, 1, 1, 1), (1 << 22, 2, 1, 1),
    (70001, 1, 64, 6), (61 * 4093, 61, 64, 6)])
def test_long_groups_of_the_loss(launches, n, g, e, k):
    status, noted = launches(LOSS.format(n=n, g=g, e=e, k=k))
    assert status == V.VMOE_OK
    fits(noted)


BACKWARD = """
    s = Norm({n}, {g}, {d}, 1, 1, 0, 2, 2, 1e-6, 1, 1, 0)
    lib.vmoe_block_norm_bwd_workspace_bytes.restype = ctypes.c_size_t
    need = lib.vmoe_block_norm_bwd_workspace_bytes(ctypes.byref(s))
    status = lib.vmoe_block_norm_bwd(ctypes.byref(s), *[FAKE] * 18, FAKE, ctypes.c_size_t(need), None)
"""


@pytest.mark.parametrize("n, g, d", [
    (1 << 23, 1 << 23, 8), (1 << 24, 1 << 24, 8), ((1 << 24) + 3, (1 << 24) + 3, 64),
    (1 << 24, 1 << 24, 256), (1 << 25, 1 << 24, 512), (1 << 22, 1 << 22, 1024),
    (1 << 28, 1 << 28, 8), (1 << 30, 1, 8), (1 << 30, 1 << 20, 32), (1 << 20, 1, 16384)])
def test_groups_of_the_norms_backward(launches, n, g, d):
    status, noted = launches(BACKWARD.format(n=n, g=g, d=d))
    assert status == V.VMOE_OK
    fits(noted)
    rows = [b for b, t in noted if t != 1024 or d > 8192]  # the others add partial rows
    assert sum(rows) >= max(g, 256)


FORWARD = """
    s = Norm({n}, {g}, {d}, 1, 1, 0, 2, 2, 1e-6, 1, 1, 0)
    status = lib.vmoe_block_norm_fwd(ctypes.byref(s), *[FAKE] * 12, None)
"""


@pytest.mark.parametrize("n, g, d", [(1 << 30, 1 << 30, 8), (1 << 30, 1, 8), (1 << 24, 2, 16384)])
def test_rows_of_the_norms_forward(launches, n, g, d):
    status, noted = launches(FORWARD.format(n=n, g=g, d=d))
    assert status == V.VMOE_OK
    fits(noted)


VALUES = """
    status = lib.vmoe_adamw_state_values(FAKE, FAKE, 1, L({n}), FAKE, {dtype}, None)
"""


@pytest.mark.parametrize("dtype", [V.VMOE_F32, V.VMOE_BF16])
@pytest.mark.parametrize("n", [1, 4096, (1 << 36) - 4096, (1 << 36) - 4095, (1 << 36) - 1])
def test_values_of_states(launches, n, dtype):
    status, noted = launches(VALUES.format(n=n, dtype=dtype))
    assert status == V.VMOE_OK
    fits(noted)
    assert sum(b for b, _ in noted) == -(-n // 4096)


@pytest.mark.parametrize("chunks", [1, 1 << 20, (1 << 20) + 1, (1 << 28) - 1])
def test_chunks_of_adamw(launches, chunks):
    text = """
        class Hyper(ctypes.Structure):
            _fields_ = [(k, D) for k in "lr b1 b2 eps scale".split()] + \\
                [("step", L), ("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]
        h = Hyper(1e-3, 0.9, 0.99, 1e-8, 1, 1, 0, 0)
        status = lib.vmoe_adamw(FAKE, L({n}), ctypes.byref(h), None, None) or \\
            lib.vmoe_grad_norm(FAKE, L({n}), D(1), D(1), FAKE, FAKE, MOST, None)
    """.format(n=chunks)
    status, noted = launches(text)
    assert status == V.VMOE_OK
    fits(noted)
    assert sum(b for b, t in noted if t == 128) == 16 * chunks
