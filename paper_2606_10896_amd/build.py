"""Builds ``libflashgmm.so`` (the HIP library, gfx950) in place next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("flashgmm.hip", "kvcache.hip")]
LIB = os.path.join(HERE, "libflashgmm.so")
INCLUDE = os.path.join(ROOT, "include")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    # packed fp32 VALU instructions are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cand = os.path.join(rocm, "bin", "hipcc")
    return cand if os.path.exists(cand) else "hipcc"


def _compile(src: str, obj: str) -> str:
    """Compiles one source; returns what the compiler printed."""
    res = subprocess.run([hipcc(), *HIPCC_FLAGS, "-I", INCLUDE, "-c", "-o", obj, src],
                         capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"hipcc failed compiling {os.path.basename(src)}")
    return res.stderr


def build(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory() as tmpdir:
        objs = [os.path.join(tmpdir, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(len(SOURCES)) as pool:
            printed = list(pool.map(_compile, SOURCES, objs))
        tmp = LIB + ".tmp"
        res = subprocess.run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp,
                              *objs], capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError("hipcc failed linking libflashgmm.so")
    if verbose:
        sys.stderr.write("".join(printed) + res.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
