"""Build libsfcgemm.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2601_16294_amd.build

Each source is compiled to an object in _build/ (in parallel), then linked
into paper_2601_16294_amd/libsfcgemm.so.  The Python binding's argument checks
(csrc/sfc_args.cpp, host code against torch's headers) become _sfcargs.so beside it.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libsfcgemm.so")
# longest first
SOURCES = ["sfc_gemm_256x256_f32.hip", "sfc_gemm_256x256_bf16.hip", "sfc_gemm_256x128.hip", "sfc_gemm_128x256.hip",
           "sfc_gemm_f8_256x256.hip", "sfc_gemm_f8_128x256.hip", "sfc_gemm_128x128.hip", "sfc_gemm_general.hip",
           "sfc_gemm.hip", "sfc_small.hip", "sfc_order.hip",
           "sfc_reduce.hip", "sfc_probe.hip", "sfc_mx4_gemm_256x256.hip", "sfc_mx4_gemm_128x128.hip", "sfc_mx4_rows.hip",
           "sfc_mx4_quant.hip", "sfc_moe.hip", "sfc_model.cpp", "sfcgemm_api.cpp", "sfc_ops_api.cpp"]
ARGS = os.path.join(PKG, "_sfcargs.so")
ARCH = "gfx950"


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def common_flags():
    return ["-x", "hip", f"--offload-arch={ARCH}", "-O3", "-std=c++20", "-fPIC",
            "-ffp-contract=off",
            # keep the compiler from forming packed fp32 instructions
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
            f"-I{INCLUDE}", f"-I{CSRC}"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [hipcc()] + common_flags() + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stderr}")
    return obj


def _build_args() -> None:
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = ARGS + ".tmp%d" % os.getpid()
    cmd = [os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-o", tmp,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", f"-I{INCLUDE}",
           f"-isystem{sysconfig.get_paths()['include']}"] + [f"-isystem{d}" for d in include_paths()]
    cmd += [os.path.join(CSRC, "sfc_args.cpp"), f"-L{libs}", f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"build of {os.path.basename(ARGS)} failed:\n{r.stderr}")
    os.replace(tmp, ARGS)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        args = ex.submit(_build_args)
        objs = list(ex.map(_compile, SOURCES))
        args.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
