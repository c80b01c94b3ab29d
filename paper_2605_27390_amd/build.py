"""Build the HIP library (libevospec.so) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libevospec.so")
SOURCES = ["kernels.hip", "gemm.hip", "tile.hip", "narrow.hip", "klgate.hip", "noalloc.hip", "kvcache.hip", "attention.hip", "sample.hip",
           "lora.hip", "kdloss.hip", "adamw.hip", "api.cpp", "decode.cpp", "adapt.cpp", "arc.cpp", "path_a.cpp"]
OBJECTS = os.path.join(HERE, "_build")
HEADERS = ["plan.hpp", "launch.hpp", "common.hpp", "slab.hpp", "slab_epilogue.hpp", "decode.hpp", "adapt.hpp", os.path.join(ROOT, "include", "evospec.h"),
           os.path.join(ROOT, "include", "evospec_arc.h"), os.path.join(ROOT, "include", "evospec_decode.h"),
           os.path.join(ROOT, "include", "evospec_adapt.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in HEADERS]
    return any(os.path.getmtime(p) > t for p in deps)


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 target feature and says so: harmless
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        sys.stderr.write(err + "\n")
        raise RuntimeError("hipcc failed")
    if verbose and err.strip():
        print(err)


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 into libevospec.so (cross-compiles without a GPU), the sources side by side;
    without `force` only those that are newer than their object, or all after a change to a header."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJECTS, exist_ok=True)
    headers = max(os.path.getmtime(h if os.path.isabs(h) else os.path.join(CSRC, h)) for h in HEADERS)

    def compile_one(source):
        src, obj = os.path.join(CSRC, source), os.path.join(OBJECTS, source + ".o")
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(headers, os.path.getmtime(src), os.path.getmtime(__file__)):
            _run([hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj + ".tmp"], verbose)
            os.replace(obj + ".tmp", obj)
        return obj

    with ThreadPoolExecutor(max(1, min(8, os.cpu_count() or 1))) as pool:
        objects = list(pool.map(compile_one, SOURCES))
    _run([hipcc, *HIPCC_FLAGS, "-shared", *objects, "-o", LIB + ".tmp"], verbose)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
