"""Build libecho.so (HIP kernels for gfx950 + host loader) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libecho.so")
ARCH = "gfx950"

# -packed-fp32-ops: keep the compiler from emitting packed FP32 VALU forms.
# atomic optimizer off: the kernels' same-address atomics already come from one lane
# (arrival counts), and the optimizer's lane-count prologue only lengthens the barrier path.
DEVICE_FLAGS = ["--offload-arch=" + ARCH, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"]
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-I", INCLUDE, "-I", CSRC]


SOURCES = ("echo_kernels.hip", "echo_norm.hip", "echo_embed.hip", "echo_loss.hip", "echo_host.cpp", "echo_ops_host.cpp")


def _run(cmds, verbose):
    """Run the commands side by side; raise if one of them fails."""
    running = []
    for cmd in cmds:
        if verbose:
            print(" ".join(cmd), flush=True)
        running.append((cmd, subprocess.Popen(cmd)))
    failed = [(cmd, p.returncode) for cmd, p in running if p.wait()]
    if failed:
        raise subprocess.CalledProcessError(failed[0][1], failed[0][0])


def build(verbose: bool = False) -> str:
    """Compile every source and link libecho.so; always rebuilds."""
    os.makedirs(BUILD, exist_ok=True)
    objects = {src: os.path.join(BUILD, os.path.splitext(src)[0] + ".o") for src in SOURCES}
    _run([["hipcc", "-c", *(DEVICE_FLAGS if src.endswith(".hip") else []), *COMMON, os.path.join(CSRC, src), "-o", obj]
          for src, obj in objects.items()], verbose)
    tmp = LIB + ".tmp"
    _run([["hipcc", "-shared", "-fPIC", "--offload-arch=" + ARCH, *objects.values(), "-o", tmp]], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
