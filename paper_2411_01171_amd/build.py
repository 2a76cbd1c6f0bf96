"""Builds the HIP library (libsi.so) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libsi.so")
SOURCES = ("si_api.hip", "si_attn_ops.hip")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-fp32 instruction forms are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the fused kernels rely on full unrolling so that every register array keeps constant indices
    "-mllvm", "-pragma-unroll-threshold=262144",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
]


def build_library(verbose: bool = False) -> str:
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    with tempfile.TemporaryDirectory(prefix="si_build_") as tmp:
        jobs = []
        for name in SOURCES:  # compiled side by side
            obj = os.path.join(tmp, name + ".o")
            cmd = [hipcc, *HIPCC_FLAGS, "-c", os.path.join(CSRC, name), "-o", obj]
            jobs.append((obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        lines, failed = [], False
        for _, job in jobs:
            out, _ = job.communicate()
            lines += out.splitlines()
            failed = failed or job.returncode != 0
        if not failed:
            cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *[obj for obj, _ in jobs], "-o", LIB_PATH]
            res = subprocess.run(cmd, capture_output=True, text=True)
            lines += (res.stdout + res.stderr).splitlines()
            failed = res.returncode != 0
    lines = [l for l in lines if "is not a recognized feature for this target" not in l]
    if failed:
        raise RuntimeError("hipcc failed:\n" + "\n".join(lines))
    if verbose and lines:
        print("\n".join(lines))
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
