"""Compile the HIP kernels and the C-ABI layer into libswiftspec.so (gfx950).

Every source is compiled by hipcc for gfx950 only; objects go to _build/
and are linked into _build/libswiftspec.so.  Packed-fp32 instruction
selection is disabled for the device code.
"""
import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libswiftspec.so")
SOURCES = ["w4a16_gemm.hip", "tree_attention.hip", "small_kernels.hip", "lm_head.hip", "w4a16_gemm_valu.hip", "greedy_accept.hip", "draft_expand.hip", "mx4_quant.hip",
           "mx4_gemm.hip", "product.hip", "fp8_quant.hip", "fp8_gemm.hip", "moe_route.hip", "moe_route_scored.hip", "draft_tree.cpp",
           "swiftspec_api.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(HERE, "..", "include")]


# per-source flags: the attention kernels keep their matrix-core
# accumulators in ordinary vector registers (the default accumulation-register
# form makes the compiler copy the output tiles between the two register
# files around every key tile)
# (in fp8_gemm the results of the matrix instructions go into multiply-adds, which
# read ordinary registers only)
EXTRA = {"tree_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form", "-fno-honor-nans"],
         "fp8_gemm.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj] + FLAGS + EXTRA.get(src, [])
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if verbose and err.strip():
        print(err, flush=True)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(4, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    cmd = [HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB + ".tmp"] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
