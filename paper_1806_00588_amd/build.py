"""Compile the HIP library in-tree for gfx950:  python -m paper_1806_00588_amd.build"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "lshbeam.hip")              # the decode step and the tables it looks up
DECODER_SRC = os.path.join(HERE, "csrc", "lshdecoder.hip")   # what stands around a decoder with a cache
LAYERS_SRC = [os.path.join(HERE, "csrc", f) for f in ("lshlayers.hip", "packed_rows.hip", "packed_tiles.hip")]   # a decoder's layers
LIB = os.path.join(HERE, "liblshbeam.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # keep the compiler from forming packed-fp32 VALU ops out of scalar float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    c = os.path.join(HERE, "csrc")
    return [os.path.join(c, f) for f in sorted(os.listdir(c))] + [
        os.path.join(os.path.dirname(HERE), "include", "lshbeam.h")]


def build(verbose: bool = True) -> str:
    """The translation units at the same time, then the library of all."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    units = [SRC, DECODER_SRC] + LAYERS_SRC
    objects = [tmp + ".%d.o" % i for i in range(len(units))]
    compiles = [[hipcc] + HIPCC_FLAGS + ["-c", "-o", o, src] for o, src in zip(objects, units)]
    link = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp] + objects
    try:
        if verbose:
            print("\n".join(" ".join(c) for c in compiles + [link]), flush=True)
        running = [subprocess.Popen(c) for c in compiles]
        failed = [c for c, p in zip(compiles, running) if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.check_call(link)
        os.replace(tmp, LIB)
    finally:
        for path in objects + [tmp]:
            if os.path.exists(path):
                os.remove(path)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    m = os.path.getmtime(LIB)
    return any(os.path.getmtime(s) > m for s in sources())


if __name__ == "__main__":
    build()
    sys.exit(0)
