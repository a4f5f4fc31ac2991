"""Build libvmoe.so (HIP, gfx950) and its Python extension in-tree.

    python -m paper_2608_16188_amd.build

Each source compiles on its own (in parallel) into _build/, then links into
paper_2608_16188_amd/libvmoe.so; binding.cpp becomes the Python extension
_train.so beside it. route.hip, adamw.hip and grouping.cpp (host code) are
compiled without floating-point contraction: their arithmetic is specified
operation by operation.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libvmoe.so")
BINDING = os.path.join(PKG, "_train.so")  # Python's side of vmoe_train.h and vmoe_head.h
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SOURCES = ["abi.hip", "route.hip", "moves.hip", "ffn.hip", "route_bwd.hip", "balance.hip",
           "abi_train.hip", "block_norm.hip", "gate_loss.hip", "adamw.hip", "abi_head.hip",
           "head_loss.hip", "grouping.cpp"]
COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
PER_FILE = {"route.hip": ["-ffp-contract=off"], "grouping.cpp": ["-ffp-contract=off"],
            "adamw.hip": ["-ffp-contract=off"]}


def _torch_flags() -> tuple[list[str], list[str]]:
    """Compiler and linker flags of an extension that reads torch tensors."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"], "/opt/rocm/include"]
    flags = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    return flags + [f"-I{p}" for p in include], [
        f"-L{libs}", "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    procs = []
    objs = []
    compile_flags, link_flags = _torch_flags()
    binding = os.path.join(BUILD, "binding.o")

    def start(src, cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))

    for src in SOURCES:
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        start(src, [HIPCC, *COMMON, *PER_FILE.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    start("binding.cpp", ["g++", *compile_flags, "-c", os.path.join(CSRC, "binding.cpp"), "-o",
                          binding])
    failed = []
    for src, p in procs:
        out = p.communicate()[0].decode(errors="replace")
        out = "\n".join(line for line in out.splitlines() if "packed-fp32-ops" not in line)
        if out.strip() and (verbose or p.returncode):
            print(f"[{src}]\n{out}", file=sys.stderr)
        if p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"hipcc failed for {failed}")
    tmp = LIB + ".tmp"
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    tmp = BINDING + ".tmp"
    subprocess.check_call(["g++", "-shared", binding, "-o", tmp, f"-L{PKG}", "-l:libvmoe.so",
                           "-Wl,-rpath,$ORIGIN", *link_flags])
    os.replace(tmp, BINDING)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
