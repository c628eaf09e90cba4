"""Build libdedloc.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2106_10207_amd.build

Flags:
  -ffp-contract=off    no implicit fused multiply-add: the library's
                       arithmetic is pinned operation by operation
  -packed-fp32-ops off no v_pk_*_f32 instructions in generated code
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdedloc.so")
SOURCES = ["kernels.hip", "ortho.hip", "embed.hip", "block.hip", "block_f32.hip", "block_f32_fp16.hip",
           "block_f32_bf16.hip", "block_fp16.hip", "block_bf16.hip", "api.hip", "api_ops.hip", "api_block.hip"]
HOST_SOURCES = ["balance.cpp"]  # host-only C++ (no device code)
ARCH = "gfx950"

HIP_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"),
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library; returns its path."""
    cc = hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, cmds = [], []
    for src in SOURCES:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmds.append([cc, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    if verbose:
        print("\n".join(" ".join(c) for c in cmds), flush=True)
    running = [subprocess.Popen(c) for c in cmds]  # side by side: the kernels' files take a minute each
    for p in running:
        p.wait()
    for p, cmd in zip(running, cmds):
        if p.returncode:
            raise subprocess.CalledProcessError(p.returncode, cmd)
    for src in HOST_SOURCES:
        obj = os.path.join(objdir, src.replace(".cpp", ".o"))
        cmd = ["g++", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wextra", "-Werror",
               "-I", os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
        objs.append(obj)
    tmp = LIB + ".tmp"
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
