"""Compile libmlda.so for gfx950 with hipcc (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libmlda.so")
SOURCES = ["mlda.hip", "operators.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # every fp64 product and sum rounds as written (parity with the fp64 definition)
    "-ffp-contract=off",
    # no packed-fp32 instruction forms
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    """Always compiles, the sources side by side; returns the library path."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as objects:
        running, linked = [], []
        for source in SOURCES:
            linked.append(os.path.join(objects, source + ".o"))
            cmd = [hipcc, *HIPCC_FLAGS, "-c", "-o", linked[-1], os.path.join(CSRC, source)]
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, subprocess.Popen(cmd)))
        for cmd, process in running:
            if process.wait():
                for _, other in running:
                    other.wait()
                raise subprocess.CalledProcessError(process.returncode, cmd)
        cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-o", LIB_PATH, *linked, "-lpthread"]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
    return LIB_PATH
