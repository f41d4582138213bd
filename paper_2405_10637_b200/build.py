"""Compile the native code in-tree: paper_2405_10637_b200/liblckv.so (CUDA, sm_100a only) and _lckv_calls.so (the
per-layer calls on torch tensors, C++)."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblckv.so")
CALLS = os.path.join(HERE, "_lckv_calls.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def sources():
    out = []
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for f in sorted(os.listdir(root)):
            if f.endswith((".cu", ".cuh", ".h")):
                out.append(os.path.join(root, f))
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    srcs = sources()
    if not force and os.path.exists(LIB) and all(
            os.path.getmtime(LIB) >= os.path.getmtime(s) for s in srcs):
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-Xlinker", "-soname=liblckv.so", "-o", tmp,
           os.path.join(CSRC, "lckv_api.cu")]
    if verbose:
        cmd[1:1] = ["-Xptxas", "-v"]
    extra = os.environ.get("LCKV_NVCC_FLAGS", "").split()   # e.g. tuning macros: -DLCKV_ALU_SLOTS=3
    cmd[1:1] = extra
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


def build_calls(force: bool = False) -> str:
    """_lckv_calls.so, linked against liblckv.so beside it and torch's libraries."""
    lib = build()
    src = os.path.join(CSRC, "lckv_calls.cpp")
    header = os.path.join(os.path.dirname(HERE), "include", "lckv.h")
    if not force and os.path.exists(CALLS) and all(os.path.getmtime(CALLS) >= os.path.getmtime(s) for s in (src, header)):
        return CALLS
    import torch
    root = os.path.dirname(torch.__file__)
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-o", tmp, src,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
           "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include"),
           lib, "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
           "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + os.path.join(root, "lib")]
    subprocess.run(cmd, check=True)
    os.replace(tmp, CALLS)
    return CALLS


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_calls(force="--force" in sys.argv))
