"""build() takes no library in which a kernel behind the pruning has a stack frame (read from the compiler's output; no GPU needed)."""
import os

import pytest

from paper_2605_00392_b200 import build

LINES = """ptxas info    : 0 bytes gmem
ptxas info    : Compiling entry function '_ZN3rtp%d%s' for 'sm_100a'
ptxas info    : Function properties for _ZN3rtp%d%s
    %d bytes stack frame, %d bytes spill stores, 0 bytes spill loads
ptxas info    : Used 128 registers, used 1 barriers
"""


def _log(frames):
    return "".join(LINES % (len(k), k, len(k), k, n, n) for k, n in frames)


def test_figures_are_read():
    log = _log([("attend_rows_kernelILi128ELi8EEEv", 0), ("sinkhorn_rows_kernelEv", 304)])
    assert build.stack_frames(log) == {"_ZN3rtp32attend_rows_kernelILi128ELi8EEEv": 0, "_ZN3rtp22sinkhorn_rows_kernelEv": 304}


@pytest.mark.parametrize("kernel", build.NO_STACK)
def test_a_stack_frame_is_refused(kernel):
    sound = [(k + "IfEEv", 0) for k in build.NO_STACK] + [("sinkhorn_rows_kernelEv", 304)]
    build.check_stack(_log(sound))
    with pytest.raises(RuntimeError, match="stack frame in " + kernel):
        build.check_stack(_log(sound + [(kernel + "I13__nv_bfloat16EEv", 8)]))
    with pytest.raises(RuntimeError, match="no figures for " + kernel):
        build.check_stack(_log([f for f in sound if kernel not in f[0]]))


def test_every_kernel_of_these_sources_is_named():
    named = set()
    for name in ("pages.cu", "rope.cu", "attend.cu", "attend_rows.cuh", "attend_tiles.cuh"):
        text = open(os.path.join(build.CSRC, name)).read().split("__global__")[1:]
        named |= {part[:part.index("_kernel(") + 7].split()[-1].split("\n")[-1] for part in text}
    assert named == set(build.NO_STACK)


def test_a_refused_library_is_not_kept(tmp_path, monkeypatch):
    lib, nvcc = tmp_path / "lib.so", tmp_path / "nvcc"
    lib.write_text("as it was")
    nvcc.write_text("#!/bin/sh\nwhile [ $# -gt 0 ]; do [ \"$1\" = -o ] && echo new > \"$2\"; shift; done\ncat %s\n" % (tmp_path / "log"))
    nvcc.chmod(0o755)
    monkeypatch.setattr(build, "LIB", str(lib))
    monkeypatch.setenv("NVCC", str(nvcc))
    frames = [(k + "Ev", 0) for k in build.NO_STACK]
    (tmp_path / "log").write_text(_log(frames + [("attend_tiles_kernelILi64EEEv", 8)]))
    with pytest.raises(RuntimeError):
        build.build(force=True)
    assert lib.read_text() == "as it was" and sorted(p.name for p in tmp_path.iterdir()) == ["lib.so", "log", "nvcc"]
    (tmp_path / "log").write_text(_log(frames))
    assert build.build(force=True) == str(lib) and lib.read_text() == "new\n"
