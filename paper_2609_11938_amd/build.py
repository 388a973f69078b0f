"""Build libopattr.so for gfx950 with hipcc, and the attention operators' Python
binding with the host compiler (in-tree, under _build/)."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(OUT_DIR, "libopattr.so")
BIND = os.path.join(OUT_DIR, "attn_bind.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = os.environ.get("OPATTR_ARCH", "gfx950")

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", f"--offload-arch={ARCH}",
    # packed fp32 instructions are disabled for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _run(cmd, out, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(out + ".tmp", out)


def build(verbose: bool = False) -> str:
    """The library, then the binding that calls it (always recompiles)."""
    build_library(verbose)
    build_binding(verbose)
    return LIB


def build_library(verbose: bool = False) -> str:
    """Compile every HIP source into one shared library; needs nothing of torch."""
    os.makedirs(OUT_DIR, exist_ok=True)
    include = os.path.join(HERE, "..", "include")
    _run(["hipcc", *FLAGS, "-I", include, "-o", LIB + ".tmp", *sources()], LIB, verbose)
    return LIB


def build_binding(verbose: bool = False) -> str:
    """Compile the attention operators' binding against the installed torch."""
    import torch

    home = os.path.dirname(torch.__file__)
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
          "-DUSE_ROCM=1", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
          *[f for d in (os.path.join(home, "include"),
                        os.path.join(home, "include", "torch", "csrc", "api", "include"),
                        os.path.join(ROCM, "include"), sysconfig.get_paths()["include"])
            for f in ("-isystem", d)],
          os.path.join(CSRC, "attn_bind.cpp"), "-o", BIND + ".tmp",
          "-L", os.path.join(home, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu",
          "-ltorch_python", "-L", OUT_DIR, "-lopattr", "-Wl,-rpath,$ORIGIN"], BIND, verbose)
    return BIND


if __name__ == "__main__":
    print(build(verbose=True))
