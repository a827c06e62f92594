"""Builds libxpress.so (the C-ABI library) in-tree with nvcc for sm_103a.

Each CUDA translation unit is compiled in parallel, then linked into
``paper_2608_02438_gb300/_build/libxpress.so``; beside it ``xpress_torch.so``,
the argument checks of the binding's torch calls (``csrc/torch_ext.cpp``, host
code against torch's headers; left out where torch is not installed).  No GPU is
needed to build.
"""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libxpress.so")
SOURCES = ["refine_kernels.cu", "read_tc.cu", "read_tcv.cu", "refine_small.cu", "pre_tc.cu", "accept_kernels.cu", "xpress_host.cu",
           "accept_noalloc.cu", "lm_head.cu", "trans_tc.cu", "train_read.cu", "train_gemm.cu",
           "train_kernels.cu", "train_host.cu", "rmsnorm.cu", "quant_fp8.cu", "matmul_fp8.cu",
           "matmul_fp8_wide.cu", "logits.cu"]
EXT = os.path.join(BUILD, "xpress_torch.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _flags():
    return ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                   "-I" + CSRC]


def _cxx() -> str:
    for cand in (os.environ.get("CXX"), shutil.which("g++"), shutil.which("c++")):
        if cand:
            return cand
    raise RuntimeError("no C++ compiler found")


def _ext_flags():
    """Compile and link flags of xpress_torch.so; None without torch."""
    import sysconfig

    try:
        import torch
    except ModuleNotFoundError as e:
        if e.name != "torch":
            raise
        return None
    t = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(nvcc()))
    inc = [os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(cuda, "include"), os.path.join(ROOT, "include")]
    lib = os.path.join(t, "lib")
    return (["-O2", "-std=c++17", "-fPIC"] + ["-I" + i for i in inc],
            ["-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
             "-L" + BUILD, "-Wl,-rpath,$ORIGIN", "-lxpress"])


def _stale(outputs, inputs):
    if not all(os.path.exists(o) for o in outputs):
        return True
    newest_in = max(os.path.getmtime(i) for i in inputs)
    return min(os.path.getmtime(o) for o in outputs) < newest_in


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    headers = [os.path.join(CSRC, h) for h in os.listdir(CSRC) if h.endswith((".cuh", ".h"))]
    headers.append(os.path.join(ROOT, "include", "xpress.h"))
    objs = []
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale([o], [s] + headers):
            jobs.append([nvcc()] + _flags() + ["-c", s, "-o", o])
    ext_src, ext_obj = os.path.join(CSRC, "torch_ext.cpp"), os.path.join(BUILD, "torch_ext.o")
    if force or _stale([ext_obj], [ext_src, os.path.join(ROOT, "include", "xpress.h")]):
        flags = _ext_flags()
        if flags:
            jobs.append([_cxx()] + flags[0] + ["-c", ext_src, "-o", ext_obj])
    if jobs:
        def run(cmd):
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError("compilation failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
            if verbose and (r.stdout or r.stderr):
                print(r.stdout + r.stderr)
        with ThreadPoolExecutor(max_workers=len(jobs)) as ex:
            list(ex.map(run, jobs))
    if force or jobs or _stale([LIB], objs):
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = [nvcc()] + ARCH + ["-shared", "-o", tmp] + objs + ["-lcudart"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
        os.replace(tmp, LIB)
    flags = _ext_flags() if force or _stale([EXT], [ext_obj, LIB]) else None
    if flags:
        tmp = EXT + f".tmp{os.getpid()}"
        r = subprocess.run([_cxx(), "-shared", "-o", tmp, ext_obj] + flags[1], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
        os.replace(tmp, EXT)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose=True))
