"""Compile libwise.so for gfx950 in-tree with hipcc.

    python -m paper_2609_27373_amd.build

Every HIP source under csrc/ is compiled, eight at a time, into one shared library next to this
file.  The packed-fp32 feature is disabled for device code; hipcc's host pass
prints a harmless warning that it does not know the feature.
"""

from __future__ import annotations

import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libwise.so")
ARCH = os.environ.get("WISE_OFFLOAD_ARCH", "gfx950")


def sources():
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


def command(out=LIB):
    return (["/opt/rocm/bin/hipcc", "-parallel-jobs=8", f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-shared",
             "-fPIC", "-Wall", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
            + sources() + ["-o", out])


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    cmd = command(tmp)
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(ln for ln in res.stderr.splitlines() if noise not in ln)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
