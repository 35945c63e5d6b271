"""Build libpowergossip.so in-tree with hipcc for gfx950 (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpowergossip.so")
SOURCES = ["pg_api.hip", "pg_edge.hip", "pg_sweep.hip", "pg_linear.hip", "pg_norm.hip", "pg_distill.hip", "pg_attention.hip", "pg_attention_backward.hip", "pg_plan.cpp"]
DEPS = SOURCES + ["pg_kernels.hip", "pg_device.h", "pg_launch.h", "pg_desc.h", "pg_plan.hpp", "pg_rows.h", "pg_attention.h",
                  os.path.join("..", "..", "include", "powergossip.h")]


def up_to_date() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(os.path.join(CSRC, d)) <= t for d in DEPS)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             # packed fp32 instructions are kept out of the generated code
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wall", "-Wno-unused-result"]
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, s + ".o") for s in SOURCES]
        cmds = [[hipcc] + flags + ["-x", "hip", "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
        if verbose:
            print("\n".join(" ".join(c) for c in cmds), flush=True)
        procs = [subprocess.Popen(c) for c in cmds]
        failed = [c for c, p in zip(cmds, procs) if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-o", LIB] + objs, check=True)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose=True)
    print(LIB)
