"""Builds libmsd.so (HIP, gfx950) in-tree with hipcc."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["k_logits.hip", "k_gemm.hip", "k_mx.hip", "msd_api.hip", "k_feature.hip", "k_attn.hip",
           "k_rows.hip", "k_tree.hip", "k_sample.hip", "k_train.hip"]
LIB = os.path.join(HERE, "libmsd.so")
ARCH = os.environ.get("MSD_OFFLOAD_ARCH", "gfx950")


def compile_one(src, verbose=False):
    obj = os.path.join(CSRC, src.replace(".hip", ".o"))
    cmd = ["hipcc", f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-c",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-result", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd, stderr=None if verbose else subprocess.DEVNULL
                          if os.environ.get("MSD_QUIET_BUILD") else None)
    return obj


def build(verbose=False):
    with ThreadPoolExecutor(4) as pool:  # the longest first
        objs = list(pool.map(lambda s: compile_one(s, verbose), SOURCES))
    cmd = ["hipcc", f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB] + objs + ["-lrocblas"]
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
