"""Builds libpcl_dnn.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _pcl_calls.so (compiled marshalling of
binding.py's smallest calls) with g++."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpcl_dnn.so")
SOURCES = ["pcl_api.cu", "tc_fprop.cu", "tc_wgrad.cu", "generic_conv.cu", "elementwise.cu", "noalloc.cu",
           "tc_gemm16.cu", "embedding.cu", "vocab_loss.cu", "orthogonalize.cu", "orthogonalize_narrow.cu",
           "rms_norm.cu", "fc_q8.cu", "grad_norm.cu", "sample_tokens.cu"]
HEADERS = ["pcl_internal.h", "pcl_ptx.cuh", "gemm16_device.cuh", os.path.join("..", "..", "include", "pcl_dnn.h")]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC"]


CALLS_SOURCE = os.path.join(CSRC, "fast_calls.cpp")
CALLS = os.path.join(HERE, "_pcl_calls.so")
CALLS_STAMP = os.path.join(HERE, "_build", "pcl_calls_built_for")


def calls_built_for() -> str:
    """What _pcl_calls.so depends on besides its sources: it holds this in `built_for`, and is used with nothing else."""
    import torch
    return f"{sys.implementation.cache_tag} torch-{torch.__version__}"


def build_calls(force: bool = False) -> str:
    deps = [CALLS_SOURCE, os.path.join(CSRC, "..", "..", "include", "pcl_dnn.h"), os.path.abspath(__file__)]
    built_for = calls_built_for()
    if not force and os.path.exists(CALLS) and all(os.path.getmtime(d) <= os.path.getmtime(CALLS) for d in deps):
        try:
            with open(CALLS_STAMP) as f:
                if f.read() == built_for:
                    return CALLS
        except OSError:
            pass
    import sysconfig

    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(NVCC))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DPCL_BUILT_FOR="{built_for}"',
           f"-I{home}/include", f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}/include", CALLS_SOURCE, f"-L{home}/lib", "-lc10", "-lc10_cuda",
           "-ltorch_cpu", "-ltorch_python", f"-Wl,-rpath,{home}/lib", "-o", CALLS]
    if os.path.exists(CALLS):
        os.remove(CALLS)                                       # (one of older sources must not stay where this fails)
    subprocess.run(cmd, check=True)
    os.makedirs(os.path.dirname(CALLS_STAMP), exist_ok=True)
    with open(CALLS_STAMP, "w") as f:
        f.write(built_for)
    return CALLS


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    try:
        build_calls(force)
    except (OSError, subprocess.CalledProcessError) as e:      # (no g++, no headers of Python or torch: binding.py does without)
        print(f"{CALLS} was not built, binding.py checks all calls itself: {e}", file=sys.stderr)
    if not force and not needs_build():
        return LIB
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(objdir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [NVCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip() and (verbose or p.returncode != 0):
            print(f"--- {src}\n{out}", file=sys.stderr)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([NVCC, "-shared", "-o", LIB, *objs], check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
