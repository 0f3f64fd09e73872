"""Build libdecomoe.so in-tree with nvcc for sm_103a, and the _marshal extension.

Each CUDA translation unit compiles in parallel (one -gencode), the plain-C
prefix selection with gcc, the Python extension that marshals the decode step's
calls with g++ against torch's headers, and the two shared libraries are linked
next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libdecomoe.so")
EXT = os.path.join(HERE, "_marshal.so")

CU_SOURCES = ["api.cu", "route.cu", "dispatch.cu", "expert_gemm.cu", "combine_compact.cu", "calib_gate.cu", "layer.cu", "decode_layer.cu", "attention.cu",
              "paged.cu", "paged_attention.cu", "paged_q4.cu", "paged_attention_q4.cu", "add_norm.cu", "w4_linear.cu", "logprobs.cu"]
C_SOURCES = ["prefix.c"]
EXT_SOURCE = "marshal.cpp"
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc_path() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found")
    return cand


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("command failed:\n" + " ".join(cmd) + "\n" + r.stdout)
    return r.stdout


def build(verbose: bool = False, ptxas_info: bool = False, force: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    nvcc = nvcc_path()
    srcs = [os.path.join(CSRC, s) for s in CU_SOURCES + C_SOURCES + [EXT_SOURCE]]
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")]
    hdrs.append(os.path.join(ROOT, "include", "decomoe.h"))
    if not force and os.path.exists(LIB) and os.path.exists(EXT):
        lib_t = min(os.path.getmtime(LIB), os.path.getmtime(EXT))
        if all(os.path.getmtime(p) < lib_t for p in srcs + hdrs + [__file__]):
            return LIB
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-fvisibility=hidden",
              "--expt-relaxed-constexpr", "-I" + os.path.join(ROOT, "include")]
    if ptxas_info:
        common += ["-Xptxas", "-v"]
    jobs = []
    for s in CU_SOURCES:
        obj = os.path.join(BUILD, s.replace(".cu", ".o"))
        jobs.append(([nvcc, *ARCH, *common, "-c", os.path.join(CSRC, s), "-o", obj], obj))
    for s in C_SOURCES:
        obj = os.path.join(BUILD, s.replace(".c", ".c.o"))
        cc = shutil.which("gcc") or "cc"
        jobs.append(([cc, "-O2", "-std=c11", "-fPIC", "-fvisibility=hidden", "-Wall",
                      "-I" + os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, s), "-o", obj], obj))
    torch_dir = list(importlib.util.find_spec("torch").submodule_search_locations)[0]
    cuda = os.path.dirname(os.path.dirname(nvcc))
    ext_obj = os.path.join(BUILD, "marshal.o")
    cxx = shutil.which("g++") or "c++"
    jobs.append(([cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I" + os.path.join(torch_dir, "include"),
                  "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(cuda, "include"), "-c",
                  os.path.join(CSRC, EXT_SOURCE), "-o", ext_obj], ext_obj))
    outs = []
    with cf.ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 4)) as ex:
        for out in ex.map(lambda j: _run(j[0]), jobs):
            outs.append(out)
    if verbose or ptxas_info:
        for o in outs:
            if o.strip():
                sys.stdout.write(o)
    tmp = LIB + ".tmp"
    _run([nvcc, *ARCH, "-shared", "-o", tmp, *[j[1] for j in jobs if j[1] != ext_obj], "-lcudart"])
    os.replace(tmp, LIB)
    tmp = EXT + ".tmp"
    _run([cxx, "-shared", "-o", tmp, ext_obj, "-L" + HERE, "-ldecomoe", "-L" + os.path.join(torch_dir, "lib"),
          "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, EXT)
    return LIB


if __name__ == "__main__":
    build(verbose=True, ptxas_info="-v" in sys.argv, force="-f" in sys.argv)
    print(LIB)
