"""Build libbd_attn.so for gfx950 with hipcc, in-tree (next to this file).

    python -m paper_2512_22234_amd.build

Every call recompiles: translation units are compiled in parallel into
_build/ and linked into paper_2512_22234_amd/libbd_attn.so.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbd_attn.so")
SOURCES = ["api.hip", "fwd.hip", "bwd.hip", "decode.hip", "paged.hip", "plan.hip", "rope.hip", "lce.hip", "aux.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
CFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    # hipcc would otherwise form packed fp32 instructions from plain float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"),
]


# Per-file additions.  MFMAs in their VGPR form: scores and score gradients
# are consumed by VALU code, so AGPR accumulators would be copied back every
# tile (the long-lived dK/dV accumulators are pinned to AGPRs explicitly).
# The forward kernel also drops NaN semantics (its inputs are finite or -inf,
# so fmax needs no quieting of its operands).
FILE_FLAGS = {
    "fwd.hip": ["-fno-honor-nans", "-mllvm", "-amdgpu-mfma-vgpr-form"],
    "bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "decode.hip": ["-fno-honor-nans", "-mllvm", "-amdgpu-mfma-vgpr-form"],
    "paged.hip": ["-fno-honor-nans", "-mllvm", "-amdgpu-mfma-vgpr-form"],
}


def compile_flags(src: str) -> list:
    """hipcc flags (without -c / -o) that build.py uses for csrc/<src>."""
    return [*CFLAGS, *FILE_FLAGS.get(src, [])]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *compile_flags(src), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), 8)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    # every kernel launched from host code must have its launch stub defined
    r = subprocess.run(["nm", "-u", tmp], capture_output=True, text=True)
    missing = [l.split()[-1] for l in r.stdout.splitlines() if "__device_stub__" in l]
    if missing:
        os.remove(tmp)
        raise RuntimeError(f"kernel launch stubs missing from the host objects: {missing}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
