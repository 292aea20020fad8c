"""Builds the HIP library (libtcr.so) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libtcr.so")
NATIVE_PATH = os.path.join(_HERE, "_native.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-cuda-version",
    # keep the compiler from forming packed-fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # every atomic add here is a one-lane ticket draw; the wave-level atomic optimiser would wrap it in a
    # cross-lane reduction whose read-back waits for the result at once instead of where it is used
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
]


def sources():
    return [os.path.join(d, f) for d in (CSRC, os.path.join(CSRC, "layers")) for f in sorted(os.listdir(d)) if f.endswith(".hip")]


def build_library(verbose: bool = False) -> str:
    """One object per source, side by side, and the library from them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        # the host pass does not know the device-only target feature and says so; that is harmless
        out = "\n".join(l for l in proc.stdout.splitlines() if "packed-fp32-ops" not in l)
        if proc.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + out)
        if verbose and out.strip():
            print(out, flush=True)

    with tempfile.TemporaryDirectory() as work:
        objects = [os.path.join(work, os.path.basename(s) + ".o") for s in sources()]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        with ThreadPoolExecutor(max_workers=4) as pool:
            list(pool.map(run, ([hipcc] + compile_flags + ["-c", "-o", o, s] for s, o in zip(sources(), objects))))
        run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB_PATH] + objects)
    return LIB_PATH


def build_native(verbose: bool = False) -> str:
    """The extension module behind binding.py's ordinary calls (host code only; torch's headers and libraries)."""
    import sysconfig

    import torch

    root = os.path.dirname(torch.__file__)
    rocm = os.path.dirname(os.path.dirname(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(rocm, "include"), "-isystem", sysconfig.get_paths()["include"],
           "-o", NATIVE_PATH, os.path.join(CSRC, "tcr_native.cpp"), "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if proc.returncode != 0:
        raise RuntimeError("g++ failed:\n" + proc.stdout)
    return NATIVE_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_native(verbose=True))
