"""Build the HIP library ``libm2r2.so`` for gfx950 in-tree.

    python -m paper_2502_02040_amd.build
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
SRCS = [os.path.join(PKG, "csrc", f) for f in ("runtime.hip", "kv8.hip")]
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libm2r2.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed fp32 instructions (v_pk_{add,mul,fma}_f32) anywhere
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fvisibility=hidden",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed ({r.returncode}):\n{msgs}")
    if verbose and msgs.strip():
        print(msgs)


def build(verbose: bool = False) -> str:
    """Compile every source side by side and link them."""
    inc = ["-I", INCLUDE, "-I", os.path.join(PKG, "csrc")]
    with tempfile.TemporaryDirectory(dir=PKG) as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SRCS]
        with ThreadPoolExecutor(len(SRCS)) as ex:
            list(ex.map(lambda so: _run([hipcc(), *HIPCC_FLAGS, *inc, "-c", "-o", so[1], so[0]], verbose),
                        zip(SRCS, objs)))
        out = os.path.join(tmp, os.path.basename(LIB))
        _run([hipcc(), *HIPCC_FLAGS, "-shared", "-o", out, *objs], verbose)
        os.replace(out, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
