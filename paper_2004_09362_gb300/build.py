"""Builds libgar.so (the C-ABI library) in-tree with nvcc for sm_103a.

Usage: python -m paper_2004_09362_gb300.build   (or via __graft_entry__.build())

Each translation unit compiles in parallel into _build/, then one link step writes
paper_2004_09362_gb300/libgar.so.  Rebuilds only when a source is newer than the
library.  The Python calls of the decoding operators (csrc/marshal.cpp) become
paper_2004_09362_gb300/_marshal.so, linked to it and to torch, and built again when torch or Python is another
one; without torch it is left out.  The generated fused/batched kernels are compiled later, at plan time, by
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
           "decode_mma_e4m3.cu", "decode_mma_f32.cu", "decode_mma_i8_f32.cu", "decode_mma_e4m3_f32.cu",
           "serve_mma_bf16.cu", "serve_mma_f16.cu", "serve_mma_i8.cu", "serve_mma_e4m3.cu", "serve_mma_f32.cu",
           "serve_mma_i8_f32.cu", "serve_mma_e4m3_f32.cu", "prefix.cu", "prefix_mma.cu", "weigh.cu", "evict.cu", "verify.cu"]
HEADERS = ["gar_internal.hpp", "gar_device.cuh", "decode.cuh", "decode_mma.cuh", "device_once.hpp", "cluster.cuh", "prefix.cuh", "tcgen05.cuh"]
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


def _older(target: str, sources) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in [*sources, os.path.join(INCLUDE, "gar.h"), os.path.abspath(__file__)])


def _library_stale() -> bool:
    return _older(OUT, [os.path.join(CSRC, f) for f in SOURCES + HEADERS])


def _torch_dir() -> str | None:
    spec = importlib.util.find_spec("torch")
    return list(spec.submodule_search_locations)[0] if spec else None


def _made_for() -> str:
    """What _marshal.so is compiled against beside its sources: this Python and this torch."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        return "\n".join([sys.version, _torch_dir(), f.read()])


def _marshal_stale() -> bool:
    stamp = os.path.join(BUILD, "marshal.for")
    if _older(MARSHAL, [os.path.join(CSRC, "marshal.cpp")]) or not os.path.exists(stamp):
        return True
    with open(stamp) as f:
        return f.read() != _made_for()


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds libgar.so, and where there is torch _marshal.so, when a source is newer than it (or always with
    force).  The library comes first: a failure of the other leaves it built.  Holds a file lock, so
    concurrent callers (test workers) build once."""
    import fcntl
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        library = force or _library_stale()
        marshal = _torch_dir() is not None and (force or _marshal_stale())
        if library or marshal:
            with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
                obj = ex.submit(_compile_marshal) if marshal else None
                if library:
                    _build_library(ex, verbose)
                if marshal:
                    _link_marshal(obj.result())
        return OUT


def _build_library(ex, verbose: bool) -> None:
    nvcc = _nvcc()
    libdir = _cuda_lib_dir(nvcc)
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE,
              "-Xcompiler", "-fvisibility=hidden"]

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src + ".o")
        cmd = [nvcc, *ARCH, *common, "-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cu"):
            cmd += ["-Xptxas", "-warn-spills"]
        r = _run(cmd, f"nvcc failed for {src}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr, file=sys.stderr)
        return obj

    objs = list(ex.map(compile_one, SOURCES))
    tmp = OUT + f".tmp{os.getpid()}"
    _run([nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-L", libdir, "-lnvrtc",
          "-Xlinker", "-rpath", "-Xlinker", libdir], "link failed")
    os.replace(tmp, OUT)


def _compile_marshal() -> str:
    obj = os.path.join(BUILD, "marshal.o")
    inc = os.path.join(_torch_dir(), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include")
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", inc, "-I",
          os.path.join(inc, "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
          "-I", cuda, "-I", "/usr/local/cuda/include", "-c", os.path.join(CSRC, "marshal.cpp"), "-o", obj],
         "g++ failed for marshal.cpp")
    return obj


def _link_marshal(obj: str) -> None:
    lib = os.path.join(_torch_dir(), "lib")
    tmp = MARSHAL + f".tmp{os.getpid()}"
    _run(["g++", "-shared", "-o", tmp, obj, "-L", PKG, "-lgar", "-L", lib, "-ltorch_python", "-ltorch_cpu",
          "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + lib], "link of _marshal.so failed")
    os.replace(tmp, MARSHAL)
    with open(os.path.join(BUILD, "marshal.for"), "w") as f:
        f.write(_made_for())


def _run(cmd, what: str):
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except FileNotFoundError as e:
        raise RuntimeError(f"{what}: {e}") from e
    if r.returncode != 0:
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")
    return r


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
