"""Builds the C-ABI CUDA library in-tree (nvcc, sm_100a only)."""
from __future__ import annotations

import glob
import os
import re
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libbnn_b200.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-shared",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-ffp-contract=off", "-Xcompiler", "-fvisibility=hidden",
    "--expt-relaxed-constexpr", "--threads", "0", "-Xptxas=-warn-spills",
]
# Kernels that keep accumulators, scales and requests in flight in registers and are laid out for exactly those that a thread has: a build in which one of them spills is refused.
UNSPILLED = ("k_mx_pair", "k_mx_few")


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def spilled(log: str) -> list[str]:
    """Kernels of UNSPILLED that ptxas reports as spilling, each with what it reports."""
    found = re.findall(r"spilled to local memory in function '(\S+)', (\d+) bytes spill stores, (\d+) bytes spill loads", log)
    return [f"{name}: {stores} bytes stored, {loads} loaded" for name, stores, loads in found if any(k in name for k in UNSPILLED)]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into libbnn_b200.so next to this file."""
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".%d.tmp" % os.getpid()
    cmd = [nvcc(), *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, *sources(), "-o", tmp]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + r.stdout + r.stderr)
    if spilled(r.stderr):
        os.remove(tmp)
        raise RuntimeError("registers are spilled in\n" + "\n".join(spilled(r.stderr)))
    os.replace(tmp, LIB)
    if verbose:
        print(r.stderr)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
