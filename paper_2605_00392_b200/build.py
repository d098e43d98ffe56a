"""Builds librtprune.so (the C-ABI library of CUDA kernels) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import glob
import os
import re
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librtprune.so")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v", "--threads", "4"]

# Kernels that may have no stack frame (the sources are pages.cu, rope.cu and attend.cu).  A form of attend_rows_kernel with one, and a
# chained kernel behind it, ended in an illegal memory access whose cause is not known; several of these stand a register or two from
# spilling, so the compiler's own figures decide whether a library is taken.
NO_STACK = ("page_map_kernel", "cache_write_kernel", "qk_norm_rope_kernel", "attend_rows_kernel", "attend_join_kernel", "attend_tiles_kernel")


def stack_frames(log: str) -> dict:
    """Bytes of stack of every function that `-Xptxas -v` reports."""
    return {name: int(n) for name, n in re.findall(r"Function properties for (\S+)\s*\n\s*(\d+) bytes stack frame", log)}


def check_stack(log: str) -> None:
    frames = stack_frames(log)
    for kernel in NO_STACK:
        of = {name: n for name, n in frames.items() if kernel in name}
        if not of:
            raise RuntimeError("the compiler's output has no figures for %s" % kernel)
        if any(of.values()):
            raise RuntimeError("a stack frame in %s: %s" % (kernel, {name: n for name, n in of.items() if n}))


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(PKG, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared library.  Returns its path."""
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [nvcc] + NVCC_FLAGS + ["-o", tmp] + sources()
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed (%d): %s" % (proc.returncode, " ".join(cmd)))
    try:
        check_stack(proc.stdout)
    except RuntimeError:
        os.remove(tmp)
        raise
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
