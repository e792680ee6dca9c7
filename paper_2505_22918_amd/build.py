"""Builds librettention.so in-tree with hipcc for gfx950.

    python -m paper_2505_22918_amd.build [--verbose]

The library is one shared object: the HIP kernels (csrc/*.hip) and the host
C ABI (csrc/api.cpp).  Packed-fp32 VALU instructions are disabled for device
code (-packed-fp32-ops off); hipcc's host pass warns that it does not know the
feature, which is harmless.
"""

from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librettention.so")
SOURCES = ["attn.hip", "attn_dense.hip", "elementwise.hip", "index.hip", "dynamic.hip", "norm.hip", "api.cpp"]
GRAD_SOURCES = ["attn_grad.hip"]  # beside them: LDS DMAs of its own
ARCH = "gfx950"


def hipcc():
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def command(out=LIB, extra=()):
    return [
        hipcc(),
        f"--offload-arch={ARCH}",
        "-O3",
        "-std=c++17",
        "-fPIC",
        "-shared",
        "-Wall",
        "-Wno-unused-command-line-argument",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-I", os.path.join(ROOT, "include"),
        *[os.path.join(CSRC, s) for s in SOURCES + GRAD_SOURCES],
        *extra,
        "-o", out,
    ]


def build(verbose: bool = False) -> str:
    """Compiles every source into librettention.so (always rebuilds); returns its path."""
    tmp = LIB + ".tmp"
    cmd = command(tmp)
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(
        line for line in (res.stdout + res.stderr).splitlines()
        if "packed-fp32-ops" not in line and line.strip()
    )
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{msgs}")
    if verbose and msgs:
        print(msgs, flush=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="--verbose" in sys.argv))
