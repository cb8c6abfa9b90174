"""Builds libsimsd.so for gfx950 with hipcc (in-tree, next to this file)."""

from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["simsd_attention.hip", "simsd_accept.hip", "simsd_lmhead.hip", "simsd_rotary.hip",
           "simsd_sample.hip", "simsd_chunk.hip", "simsd_window.hip", "simsd_fp4.hip", "simsd_chunk_fp4.hip",
           "simsd_verify_span.hip", "simsd_api.cpp", "simsd_ops_api.cpp", "simsd_span_api.cpp",
           "simsd_plan.cpp", "simsd_ops_plan.cpp", "simsd_span_plan.cpp"]
OUT = os.path.join(HERE, "libsimsd.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         # packed FP32 instructions are kept out of every kernel
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def build(verbose: bool = False) -> str:
    """Compile every source into libsimsd.so; returns its path."""
    objs = []
    os.makedirs(os.path.join(ROOT, "_build"), exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(ROOT, "_build", src + ".o")
        cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
        objs.append(obj)
    for cmd, p in procs:
        out, _ = p.communicate()
        msgs = [l for l in out.splitlines() if "packed-fp32-ops' is not a recognized" not in l]
        if p.returncode != 0:
            raise RuntimeError("build failed: " + " ".join(cmd) + "\n" + "\n".join(msgs))
        if verbose and msgs:
            print("\n".join(msgs), file=sys.stderr)
    tmp = OUT + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed: " + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
