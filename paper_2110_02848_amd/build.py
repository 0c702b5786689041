"""Build libfstcompose.so (HIP for gfx950) in the package directory.

The library is compiled with hipcc straight from ``csrc/``: IEEE binary32
arithmetic (no fast-math, no denormal flushing, no contraction), and packed
FP32 instructions disabled.
"""
from __future__ import annotations

import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libfstcompose.so")
SOURCES = ["primitives.hip", "compose.hip", "compose3.hip", "score.hip", "recurrence.hip",
           "head.hip", "norms.hip", "linear.hip", "window.hip", "api.cpp"]
ARCH = "gfx950"


def hipcc():
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def compile_flags():
    return [
        f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
        "-fno-gpu-flush-denormals-to-zero", "-ffp-contract=off", "-fno-fast-math",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-fvisibility=hidden", "-Wall", "-Wno-unused-function", "-Wno-unused-command-line-argument",
        # a lambda's local that shadows a variable of the enclosing function
        # leaves the outer one unset: an error, not a warning
        "-Werror=shadow-uncaptured-local",
        "-I", INCLUDE, "-I", CSRC,
    ]


def build(verbose=False):
    """Compile every source and link the shared library (always rebuilds)."""
    cc = hipcc()
    objs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src + ".o")
        cmd = [cc, *compile_flags(), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        objs.append(obj)
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    for o in objs:
        os.remove(o)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
