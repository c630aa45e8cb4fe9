"""Compile libmlda.so for gfx950 with hipcc (cross-compiles without a GPU), and _tensors.so, the operators' calls
on torch tensors, with the host compiler."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libmlda.so")
SOURCES = ["mlda.hip", "operators.hip", "mx4.hip", "training.hip"]
TENSORS_PATH = os.path.join(_HERE, "_tensors.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # every fp64 product and sum rounds as written (parity with the fp64 definition)
    "-ffp-contract=off",
    # no packed-fp32 instruction forms
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _tensors_lack() -> str | None:
    """What _tensors.so cannot be built without and is not there: the host compiler, or torch's or Python's headers."""
    compiler = os.environ.get("CXX", "g++")
    if shutil.which(compiler) is None:
        return f"no host compiler ({compiler})"
    if importlib.util.find_spec("torch") is None:
        return "no torch"
    import torch
    for header in (os.path.join(os.path.dirname(torch.__file__), "include", "ATen", "ATen.h"), os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        if not os.path.exists(header):
            return f"no {header}"
    return None


def _tensors_command(rocm: str) -> list[str]:
    """_tensors.so against torch's headers and libraries, and libmlda.so beside it."""
    import torch
    at = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
            "-DTORCH_API_INCLUDE_EXTENSION_H", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            "-isystem", os.path.join(at, "include"), "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(rocm, "include"), "-isystem", sysconfig.get_paths()["include"],
            "-o", TENSORS_PATH, os.path.join(CSRC, "tensors.cpp"), "-L" + os.path.join(at, "lib"), "-L" + _HERE, "-l:libmlda.so",
            "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + os.path.join(at, "lib")]


def build(verbose: bool = False) -> str:
    """Always compiles, the sources side by side; returns the library path.  The sampler needs libmlda.so alone: where there is nothing to
    build _tensors.so with, that is said, and the operators raise ImportError."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmds):
        running = []
        for cmd in cmds:
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, subprocess.Popen(cmd)))
        for process in [p for _, p in running]:
            process.wait()
        for cmd, process in running:
            if process.returncode:
                raise subprocess.CalledProcessError(process.returncode, cmd)

    with tempfile.TemporaryDirectory() as objects:
        linked = [os.path.join(objects, source + ".o") for source in SOURCES]
        compiled = [flag for flag in HIPCC_FLAGS if flag != "-shared"]
        run([hipcc, *compiled, "-c", "-o", o, os.path.join(CSRC, source)] for o, source in zip(linked, SOURCES))
        run([[hipcc, "--offload-arch=gfx950", "-shared", "-Wl,-soname,libmlda.so", "-o", LIB_PATH, *linked, "-lpthread"]])
    if os.path.exists(TENSORS_PATH):
        os.remove(TENSORS_PATH)                      # (calls into the library as it was before)
    lack = _tensors_lack()
    if lack:
        print(f"{TENSORS_PATH} is not built, and the operators on tensors are not there: {lack}", file=sys.stderr, flush=True)
    else:
        run([_tensors_command(os.environ.get("ROCM_PATH", "/opt/rocm"))])
    return LIB_PATH
