"""Build libckm.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libckm.so")
SOURCES = [os.path.join(HERE, "csrc", "ckm_kernels.hip"), os.path.join(HERE, "csrc", "ckm_plan.hip"),
           os.path.join(HERE, "csrc", "ckm_noalloc.hip"), os.path.join(HERE, "csrc", "ckm_tiles.hip"),
           os.path.join(HERE, "csrc", "ckm_tiles.cpp"),
           os.path.join(HERE, "csrc", "ckm_dropout.hip"), os.path.join(HERE, "csrc", "ckm_layer_norm.hip"),
           os.path.join(HERE, "csrc", "ckm_softmax.hip"), os.path.join(HERE, "csrc", "ckm_matrix.hip"),
           os.path.join(HERE, "csrc", "ckm_gated.hip"), os.path.join(HERE, "csrc", "ckm_cross_entropy.hip"),
           os.path.join(HERE, "csrc", "ckm_clip.hip"),
           os.path.join(HERE, "csrc", "ckm_host.cpp")]
ARCH = "gfx950"


def compile_command(source: str, out: str) -> list:
    return ["hipcc", "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-c",
            "-Wall", "-Wno-unused-result",
            # packed fp32 VALU ops stay off (none are needed; some forms are unreliable)
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"),
            source, "-o", out]


def _run(cmd: list, verbose: bool):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("hipcc failed building libckm.so")
    if verbose:
        sys.stderr.write(res.stderr)


def build(verbose: bool = False) -> str:
    """Compiles every source anew, a few at a time, and links them."""
    tmp = LIB_PATH + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as d:
        objects = [os.path.join(d, os.path.basename(s) + ".o") for s in SOURCES]
        with concurrent.futures.ThreadPoolExecutor(min(8, len(SOURCES))) as pool:
            for f in [pool.submit(_run, compile_command(s, o), verbose) for s, o in zip(SOURCES, objects)]:
                f.result()
        _run(["hipcc", "--offload-arch=" + ARCH, "-shared", "-fPIC", *objects, "-o", tmp], verbose)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
