"""Builds librgc.so (the gfx950 HIP library behind include/rgc.h) in-tree with hipcc.

Build-time hooks (the library itself reads no environment variable): HIPCC names another compiler driver;
RGC_EXTRA_FLAGS appends flags for tuning experiments, e.g. -DRGC_CHUNK=4096 (wave-chunk size).
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librgc.so")
OBJECTS = os.path.join(HERE, "_build")
SOURCES = ["rgc_api.cpp", "rgc_compress.hip", "rgc_decompress.hip", "rgc_threshold.hip", "rgc_yardstick.hip",
           "rgc_vocab.hip", "rgc_recurrence.hip", "rgc_embed.hip",
           "rgc_convolution.hip", "rgc_scan.hip", "rgc_scan_backward.hip", "rgc_parts.hip"]
HEADERS = ["rgc_internal.h", "rgc_device.h", "rgc_exact.h", "rgc_tickets.h", "rgc_tiles.h", "rgc_lm.h", "rgc_sequence.h", "rgc_scan.h", "rgc_stretch.h", os.path.join("..", "..", "include", "rgc.h"),
           os.path.join("..", "..", "include", "rgc_diag.h")]

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    "-ffp-contract=off",                       # the oracle is built the same way: no silent fma
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _newest(paths) -> float:
    return max(os.path.getmtime(os.path.join(CSRC, f)) for f in paths)


def needs_build() -> bool:
    return not os.path.exists(LIB) or _newest(SOURCES + HEADERS) > os.path.getmtime(LIB)


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l)   # the host pass does not know the device feature
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)


def build(force: bool = True, verbose: bool = False) -> str:
    """Compiles the sources side by side and links them.  Without `force`: those only that changed since their object was made."""
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    extra = os.environ.get("RGC_EXTRA_FLAGS", "").split()      # tuning experiments only
    os.makedirs(OBJECTS, exist_ok=True)

    def compile_one(source: str) -> str:
        target = os.path.join(OBJECTS, source + (".extra.o" if extra else ".o"))
        if force or extra or not os.path.exists(target) or _newest([source] + HEADERS) > os.path.getmtime(target):
            _run([hipcc] + FLAGS + extra + ["-x", "hip", "-c", os.path.join(CSRC, source), "-o", target], verbose)
        return target

    jobs = int(os.environ.get("MAX_JOBS", 0)) or min(16, os.cpu_count() or 1)
    with ThreadPoolExecutor(jobs) as pool:
        objects = list(pool.map(compile_one, SOURCES))
    _run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950"] + objects + ["-o", LIB], verbose)
    return LIB


if __name__ == "__main__":
    build(force="--changed" not in sys.argv[1:], verbose=True)
    print("built", LIB)
    sys.exit(0)
