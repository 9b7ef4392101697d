"""Build libspeccascade.so for gfx950 in-tree (``hipcc``, no JIT cache).

``python -m paper_2405_19261_amd.build`` compiles the kernels and the C
interface into ``paper_2405_19261_amd/libspeccascade.so``.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libspeccascade.so")
SOURCES = ["spc_kernels.hip", "spc_sample.hip", "spc_kv.hip", "spc_kv_shared.hip",
           "spc_kv_evict.hip", "spc_api.cpp"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Werror",
    "-Wno-unused-function",
    # keep float code out of the packed-FP32 VALU forms
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(out=LIB, extra=(), verbose=False):
    objs = [os.path.join(CSRC, src + ".o") for src in SOURCES]

    def compile_one(src, obj):
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        cmd = [HIPCC, *FLAGS, *extra, "-I", INCLUDE, "-I", CSRC, *lang, "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)

    with ThreadPoolExecutor(max_workers=6) as pool:
        list(pool.map(compile_one, SOURCES, objs))
    tmp = out + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    subprocess.run(cmd, check=True)
    os.replace(tmp, out)
    for o in objs:
        os.remove(o)
    return out


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
