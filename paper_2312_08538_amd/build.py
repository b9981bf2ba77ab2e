"""Builds libconef.so (HIP kernels + C ABI) for gfx950 with hipcc, and _face.so (marshalling from torch tensors, host code
only) with the host compiler, in-tree.  The library needs neither torch nor the host compiler: where these are missing it is built alone, and
the calls that go through _face.so say so when they are made."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libconef.so")
SOURCES = ["api.cpp", "plan.cpp", "kernels_generic.hip", "kernels_orth.hip", "kernels_octet.hip", "kernels_strip.hip", "kernels_ragged.hip", "kernels_mixed.hip", "kernels_mfma.hip", "kernels_pack.hip", "kernels_sketch.hip", "kernels_small.hip", "kernels_walk.hip", "layers.cpp", "kernels_norm.hip", "kernels_mx.hip", "kernels_mx_product.hip", "kernels_q8.hip", "kernels_q8_product.hip", "kernels_rms.hip", "kernels_loss.hip"]
FACE = os.path.join(HERE, "_face.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# -ffp-contract=off: the quantiser's decisions are taken in fp32 in a fixed order, every
#   fused multiply-add is written explicitly in the sources.
# packed-fp32 ops are switched off for all device code.
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function"]


def build_face(verbose: bool = False) -> str:
    import sysconfig

    import torch

    root = os.path.dirname(torch.__file__)
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "face.cpp"), "-o", FACE,
           "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return FACE


def build_library(verbose: bool = False) -> str:
    from concurrent.futures import ThreadPoolExecutor

    def compile_one(src: str) -> str:
        path = os.path.join(CSRC, src)
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = [HIPCC, *FLAGS, "-x", "hip", "-c", path, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1, 8)) as pool:
        face = pool.submit(build_face, verbose)
        objs = list(pool.map(compile_one, SOURCES))
    cmd = [HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    try:
        face.result()
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        if os.path.exists(FACE):
            os.remove(FACE)                     # another build's
        print(f"{FACE} is not built, and calls on torch tensors that need it will say so: {e}", file=sys.stderr, flush=True)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose="-v" in sys.argv))
