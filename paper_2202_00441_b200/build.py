"""Builds libfewbit.so in-tree with nvcc for sm_100a (no other target)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libfewbit.so")
TORCH_LIB = os.path.join(PKG, "_fewbit_torch.so")
OBJ_DIR = os.path.join(PKG, "build")

# (source, object stem, extra flags); the forward kernels are instantiated once per activation
SOURCES = [("fewbit_kernels.cu", "fewbit_kernels", []), ("fewbit_host.cu", "fewbit_host", []),
           ("fewbit_static.cu", "fewbit_static", []), ("fewbit_scan.cu", "fewbit_scan", []), ("fewbit_queue.cu", "fewbit_queue", []),
           ("fewbit_table.cpp", "fewbit_table", []), ("fewbit_adamw.cu", "fewbit_adamw", []),
           ("fewbit_qknorm.cu", "fewbit_qknorm", []), ("fewbit_attention.cu", "fewbit_attention", []),
           ("fewbit_attention_inst.cu", "fewbit_attention_bf16", ["-DFEWBIT_ATTN_F16=0"]),
           ("fewbit_attention_inst.cu", "fewbit_attention_f16", ["-DFEWBIT_ATTN_F16=1"])]
SOURCES += [("fewbit_fwd_inst.cu", f"fewbit_fwd_act{a}", [f"-DFEWBIT_ACT_ID={a}"]) for a in range(9)]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC,-fvisibility=hidden,-O2", "-I", INCLUDE, "-I", CSRC,
    *os.environ.get("FEWBIT_EXTRA_NVCC_FLAGS", "").split(),
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build_torch_module(force: bool = False) -> str:
    """The extension module that marshals PyTorch tensors (host code only; links libfewbit.so beside it)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    src, obj = os.path.join(CSRC, "fewbit_torch.cpp"), os.path.join(OBJ_DIR, "fewbit_torch.o")
    deps = [src, os.path.join(INCLUDE, "fewbit.h")]
    if force or _stale(obj, deps):
        includes = [*cpp_extension.include_paths("cuda"), sysconfig.get_paths()["include"], INCLUDE]
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-DTORCH_EXTENSION_NAME=_fewbit_torch",
                               "-DTORCH_API_INCLUDE_EXTENSION_H", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                               *[f for i in includes for f in ("-isystem", i)], "-c", src, "-o", obj])
    if force or _stale(TORCH_LIB, [obj]):
        tmp = TORCH_LIB + f".{os.getpid()}.tmp"
        libs = [f for d in cpp_extension.library_paths("cuda") if os.path.isdir(d) for f in ("-L", d)]
        subprocess.check_call(["g++", "-shared", "-o", tmp, obj, *libs, "-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_python",
                               "-L", PKG, "-l:libfewbit.so", "-Wl,-rpath,$ORIGIN"])
        os.replace(tmp, TORCH_LIB)
    return TORCH_LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(INCLUDE, "fewbit.h"))
    os.makedirs(OBJ_DIR, exist_ok=True)
    jobs = []
    for src, stem, extra in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(OBJ_DIR, stem + ".o")
        if force or _stale(obj, [path] + headers):
            cmd = [_nvcc(), *NVCC_FLAGS, *extra, "-c", path, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)
    with concurrent.futures.ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 4))) as pool:
        for res in pool.map(lambda c: subprocess.run(c, capture_output=True, text=True), jobs):
            if verbose and res.stderr:
                print(res.stderr)
            if res.returncode != 0:
                raise RuntimeError("nvcc failed:\n" + " ".join(res.args) + "\n" + res.stdout + res.stderr)
    objs = [os.path.join(OBJ_DIR, stem + ".o") for _, stem, _ in SOURCES]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + f".{os.getpid()}.tmp"
        subprocess.check_call([_nvcc(), "-shared", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    build_torch_module(force)
    return LIB


if __name__ == "__main__":
    import sys
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
