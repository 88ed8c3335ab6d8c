"""Builds libxenos.so (HIP kernels + C-ABI host library) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libxenos.so")
SOURCES = ["xenos_kernels.hip", "xenos_conv3.hip", "xenos_linked.hip", "xenos_unit.hip", "xenos_wave.hip", "xenos_quant.hip",
           "xenos_cache.hip", "xenos_logprobs.hip", "xenos_attention.hip", "xenos_lib.cpp", "xenos_tokens.cpp"]
HEADERS = ["kernels.h", "token_kernels.h", "token_device.h", "status.h", "device_common.h", "per_device.h", "wave_gemm.h", "index_div.h", os.path.join("..", "..", "include", "xenos.h")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build_library(force: bool = True, verbose: bool = False) -> str:
    """Compile every source with hipcc and link the shared library. Returns its path."""
    if not force and not stale():
        return LIB
    from concurrent.futures import ThreadPoolExecutor
    objs = [os.path.join(CSRC, os.path.splitext(src)[0] + ".o") for src in SOURCES]
    cmds = [["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj] for src, obj in zip(SOURCES, objs)]
    with ThreadPoolExecutor(max_workers=len(cmds)) as ex:      # one hipcc per source, side by side
        list(ex.map(lambda c: _run(c, verbose), cmds))
    _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], verbose)
    return LIB


def _run(cmd, verbose):
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("build failed: %s\n%s" % (" ".join(cmd), out))
    if verbose and out.strip():
        print(out, file=sys.stderr)


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
