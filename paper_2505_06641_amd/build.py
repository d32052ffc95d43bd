"""Builds the HIP library for gfx950 with hipcc, and, where torch is installed, the Python extension that checks the operators' tensors;
both in-tree."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libsneakpeek_hip.so")
NATIVE = os.path.join(PKG, "_ops_native.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]


def sources():
    return [os.path.join(CSRC, "sp_api.hip"), os.path.join(CSRC, "sp_ops.hip"), os.path.join(CSRC, "sp_ops_experts.hip")]


def native_command(hipcc: str):
    """Host code only: the C API of Python, torch's tensors, and the library's C entry points."""
    from torch.utils import cpp_extension
    torch_lib = cpp_extension.library_paths()[0]
    cmd = [hipcc, "-O2", "-std=c++20", "-fPIC", "-shared", "-Wall", "-Wno-unknown-pragmas",
           "-I" + os.path.join(ROOT, "include"), "-I" + sysconfig.get_paths()["include"]]
    for path in cpp_extension.include_paths():
        cmd += ["-isystem", path]
    cmd += [os.path.join(CSRC, "sp_ops_torch.cpp"), "-o", NATIVE, "-L" + torch_lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip",
            "-L" + PKG, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
    return cmd


def build_library(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    run([hipcc] + HIPCC_FLAGS + sources() + ["-o", LIB])
    if importlib.util.find_spec("torch") is not None:
        run(native_command(hipcc))
    elif verbose:
        print("no torch here: the extension of binding.Ops is not built", flush=True)
    return LIB


if __name__ == "__main__":
    build_library()
    sys.exit(0)
