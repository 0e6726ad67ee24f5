"""Build step of the HIP library: hipcc for gfx950 into ``libdelta_attn.so``.

Compiled in-tree so the shared object travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdelta_attn.so")
SOURCES = [os.path.join(CSRC, f) for f in ("da_kernels.hip", "da_api.cpp", "da_pages.hip", "da_pages8.hip", "da_select.hip",
                                          "da_paged_attn.hip", "da_paged_api.cpp", "da_pages8_api.cpp")]
ARCH = "gfx950"


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def compile_flags() -> list:
    return [
        f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
        "-Wall", "-Wno-unused-function",
        # no kernel's decisions depend on NaN, which passes through their arithmetic: lets max() skip
        # NaN quieting
        "-fno-honor-nans",
        # never let the compiler form packed fp32 VALU ops (v_pk_*_f32)
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-I", os.path.join(ROOT, "include"),
    ]


def build_library(verbose: bool = False) -> str:
    """Compiles the sources side by side and links them."""
    tmp = LIB + ".tmp"
    flags = [f for f in compile_flags() if f != "-shared"]
    with tempfile.TemporaryDirectory() as td:
        objects = [os.path.join(td, os.path.basename(s) + ".o") for s in SOURCES]
        cmds = [[hipcc()] + flags + ["-c", s, "-o", o] for s, o in zip(SOURCES, objects)]
        if verbose:
            print("\n".join(" ".join(c) for c in cmds), flush=True)
        jobs = [subprocess.Popen(c) for c in cmds]
        for job, cmd in zip(jobs, cmds):
            if job.wait():
                for other in jobs:
                    other.wait()
                raise subprocess.CalledProcessError(job.returncode, cmd)
        link = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC"] + objects + ["-o", tmp]
        subprocess.run(link, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
