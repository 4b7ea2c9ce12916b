"""Build libmsda.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

    python -m paper_2505_14022_amd.build          # -> paper_2505_14022_amd/_lib/libmsda.so
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB_DIR = os.path.join(PKG, "_lib")
LIB_PATH = os.path.join(LIB_DIR, "libmsda.so")
SOURCES = ["msda_api.cpp", "msda_arrange.cpp", "msda_fwd.hip", "msda_bwd.hip", "msda_bwd_value.hip",
           "msda_prologue.hip", "msda_noalloc.hip", "msda_layer_api.cpp", "msda_norm.hip", "msda_rotary.hip",
           "msda_attn_fwd.hip", "msda_attn_bwd.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-Wall",
    # packed fp32 (v_pk_*_f32) stays off: the compiler's packed forms are not used on this path
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics",
]


def build(verbose: bool = False) -> str:
    """Compile every source (in parallel: each is independent of the others) and link the library."""
    os.makedirs(LIB_DIR, exist_ok=True)
    tmp = LIB_PATH + ".tmp%d" % os.getpid()

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as work:
        objects = [os.path.join(work, s + ".o") for s in SOURCES]
        includes = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        compile_flags = [f for f in FLAGS if f != "-shared"]
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: run([HIPCC] + compile_flags + includes +
                                         ["-c", os.path.join(CSRC, so[0]), "-o", so[1]]), zip(SOURCES, objects)))
        run([HIPCC] + FLAGS + ["-o", tmp] + objects)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
