"""Build libsats.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

    python -m paper_2607_08991_amd.build
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libsats.so")
SOURCES = [os.path.join(CSRC, f) for f in ("sats.hip", "serve.hip", "attend.hip", "attend_prefix.hip", "attend_e4m3.hip",
                                              "attend_int8.hip")]
ARCH = "gfx950"


def hipcc() -> str:
    for c in (os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc"), shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found (ROCm is required to build the library)")


def command(out: str = LIB):
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-shared", "-fPIC",
            # packed fp32 instructions are left out of every kernel
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", os.path.join(ROOT, "include"), "-o", out] + SOURCES


def _run(cmd) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"hipcc failed with exit code {r.returncode}")


def build(verbose: bool = True) -> str:
    """Each source on its own (side by side: the kernels' instances are most of the work), then the library."""
    tmp = LIB + ".tmp"
    flags = [a for a in command(tmp) if a not in SOURCES and a not in ("-shared", "-o", tmp)]
    if verbose:
        print(" ".join(command(tmp)), flush=True)
    with tempfile.TemporaryDirectory() as folder:
        objects = [os.path.join(folder, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(len(SOURCES)) as pool:
            list(pool.map(_run, [flags + ["-c", s, "-o", o] for s, o in zip(SOURCES, objects)]))
        _run([hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objects)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build()
