"""Builds libgar.so (the C-ABI library) in-tree with nvcc for sm_103a.

Usage: python -m paper_2004_09362_gb300.build   (or via __graft_entry__.build())

Each translation unit compiles in parallel into _build/, then one link step writes
paper_2004_09362_gb300/libgar.so.  Rebuilds only when a source is newer than the
library.  The Python calls of the decoding operators (csrc/marshal.cpp) become
paper_2004_09362_gb300/_marshal.so, linked to it and to torch.  The generated fused/batched kernels are compiled later, at plan time, by
NVRTC inside the library.
"""

from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT = os.path.join(PKG, "libgar.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
BUILD = os.path.join(ROOT, "_build")

SOURCES = ["api.cpp", "plan.cpp", "codegen.cpp", "jit.cpp", "step_kernels.cu", "rope.cu", "cache.cu",
           "decode_api.cu", "decode_general.cu", "decode_mma_bf16.cu", "decode_mma_f16.cu", "decode_mma_i8.cu",
           "decode_mma_e4m3.cu", "decode_mma_f32.cu", "decode_mma_i8_f32.cu", "decode_mma_e4m3_f32.cu"]
HEADERS = ["gar_internal.hpp", "gar_device.cuh", "decode.cuh", "decode_mma.cuh", "device_once.hpp"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    p = shutil.which("nvcc")
    if p:
        return p
    cand = "/usr/local/cuda/bin/nvcc"
    if os.path.exists(cand):
        return cand
    raise RuntimeError("nvcc not found")


def _cuda_lib_dir(nvcc: str) -> str:
    root = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
    for sub in ("lib64", "lib", "targets/sbsa-linux/lib", "targets/x86_64-linux/lib"):
        d = os.path.join(root, sub)
        if os.path.exists(os.path.join(d, "libnvrtc.so")):
            return d
    return os.path.join(root, "lib64")


def _stale() -> bool:
    if not os.path.exists(OUT) or not os.path.exists(MARSHAL):
        return True
    t = min(os.path.getmtime(OUT), os.path.getmtime(MARSHAL))
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS + ["marshal.cpp"]]
    deps += [os.path.join(INCLUDE, "gar.h"), os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds libgar.so when a source is newer than it (or always with force).  Holds a
    file lock, so concurrent callers (test workers) build once."""
    import fcntl
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        if not force and not _stale():
            return OUT
        return _build(verbose)


def _build(verbose: bool) -> str:
    nvcc = _nvcc()
    libdir = _cuda_lib_dir(nvcc)
    os.makedirs(BUILD, exist_ok=True)
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE,
              "-Xcompiler", "-fvisibility=hidden"]

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src + ".o")
        cmd = [nvcc, *ARCH, *common, "-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cu"):
            cmd += ["-Xptxas", "-warn-spills"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr, file=sys.stderr)
        return obj

    def compile_marshal() -> str:
        obj = os.path.join(BUILD, "marshal.o")
        inc = os.path.join(_torch_dir(), "include")
        cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
        _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", inc, "-I",
              os.path.join(inc, "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
              "-I", cuda, "-I", "/usr/local/cuda/include", "-c", os.path.join(CSRC, "marshal.cpp"), "-o", obj],
             "g++ failed for marshal.cpp")
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        marshal = ex.submit(compile_marshal)
        objs = list(ex.map(compile_one, SOURCES))
        marshal_obj = marshal.result()
    tmp = OUT + f".tmp{os.getpid()}"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-L", libdir, "-lnvrtc",
           "-Xlinker", "-rpath", "-Xlinker", libdir]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    lib = os.path.join(_torch_dir(), "lib")
    tmp = MARSHAL + f".tmp{os.getpid()}"
    _run(["g++", "-shared", "-o", tmp, marshal_obj, "-L", PKG, "-lgar", "-L", lib, "-ltorch_python", "-ltorch_cpu",
          "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + lib], "link of _marshal.so failed")
    os.replace(tmp, MARSHAL)
    return OUT


def _torch_dir() -> str:
    return list(importlib.util.find_spec("torch").submodule_search_locations)[0]


def _run(cmd, what: str) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
