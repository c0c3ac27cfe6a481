"""Build libspd.so (the C-ABI library with the gfx950 kernels) in-tree with hipcc."""
import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libspd.so")
SOURCES = [os.path.join(PKG, "csrc", f) for f in ("spd_kernels.hip", "spd_decode.hip", "spd_prefill.hip", "spd_cache.hip",
                                                      "spd_seqattn.hip", "spd_ruleattn.hip", "spd_rope.hip", "spd_api.cpp")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions stay off: plain float code only
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result",
    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
]


def commands(out, objects):
    """A command a source, into the folder `objects`, and the one that links them to `out`."""
    objs = [os.path.join(objects, os.path.basename(s) + ".o") for s in SOURCES]
    return [[HIPCC] + FLAGS + ["-c", s, "-o", o] for s, o in zip(SOURCES, objs)], \
        [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", out]


def build(verbose=True):
    """The sources are independent of each other and compile side by side."""
    tmp = LIB + ".tmp"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as pool:
        compiles, link = commands(tmp, objects)
        list(pool.map(run, compiles))
        run(link)
    shutil.move(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
