"""Builds libheinsen_scan.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libheinsen_scan.so")
SOURCES = ["heinsen_scan.cu", "heinsen_attention.cu", "heinsen_norms.cu", "heinsen_delta.cu", "heinsen_delta_backward.cu", "heinsen_beam.cu"]
HEADERS = ["hs_device.cuh", "hs_kernels.cuh", "hs_pairs.cuh", "hs_internal.h", "ha_common.cuh", "ha_host.h", "ha_ptx.cuh", "ha_simt.cuh", "ha_mma.cuh", "hn_norms.cuh", "hd_warp.cuh",
           "hd_scan.cuh", "hd_scan_mma.cuh", "hd_grad.cuh", "hd_grad_mma.cuh", "hd_step.cuh", "hb_beam.cuh", "hd_host.h",
           os.path.join("..", "..", "include", "heinsen_scan.h"), os.path.join("..", "..", "include", "heinsen_attention.h"),
           os.path.join("..", "..", "include", "heinsen_delta.h"),
           os.path.join("..", "..", "include", "heinsen_beam.h")]
NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


DEBUG_LIB = os.path.join(_HERE, "libheinsen_scan_debug.so")


def is_stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; return its path.
    debug=True builds the checked variant (-DHEINSEN_DEBUG: index checks that record instead of trapping)
    beside the normal one."""
    lib = DEBUG_LIB if debug else LIB
    if force or is_stale(lib):
        tmp = f"{lib}.{os.getpid()}.tmp"
        with tempfile.TemporaryDirectory() as objs:  # one nvcc for each source, side by side
            compiling = []
            for src in SOURCES:
                cmd = [_nvcc(), *NVCC_FLAGS, *(["-DHEINSEN_DEBUG"] if debug else []), "-c", os.path.join(CSRC, src),
                       "-o", os.path.join(objs, src + ".o")]
                if verbose:
                    cmd[1:1] = ["-Xptxas", "-v"]
                    print(" ".join(cmd), file=sys.stderr)
                compiling.append((cmd, subprocess.Popen(cmd, cwd=CSRC)))
            failed = [cmd for cmd, proc in compiling if proc.wait() != 0]
            if failed:
                raise subprocess.CalledProcessError(1, failed[0])
            subprocess.check_call([_nvcc(), *NVCC_FLAGS, "-shared", "-o", tmp, *(cmd[-1] for cmd, _ in compiling)], cwd=CSRC)
        os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
