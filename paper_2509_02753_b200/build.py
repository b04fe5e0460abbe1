"""Builds the CUDA library in-tree: csrc/*.cu -> liblexi_moe.so (sm_100a only), and the Python module
csrc/kv_binding.cpp -> _kv_native.so that calls it (against the torch that is installed; the library needs none, and
without torch only the library is built).

nvcc cross-compiles without a GPU.  Objects go to ``_build/`` at the repository
root; a source is recompiled when it or any header is newer than its object.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJ_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "liblexi_moe.so")
NATIVE = os.path.join(PKG, "_kv_native.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC,
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(INCLUDE, "*.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)
    jobs = []
    objects = []
    for src in sources:
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        objects.append(obj)
        stale = force or not os.path.exists(obj) or \
            os.path.getmtime(obj) < max(os.path.getmtime(src), newest_header)
        if stale:
            jobs.append([_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) +
                        ["-c", src, "-o", obj])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError("compiler failed: " + " ".join(cmd))

    with ThreadPoolExecutor(max_workers=8) as pool:
        list(pool.map(run, jobs))
    if jobs or not os.path.exists(LIB):
        tmp = LIB + f".tmp{os.getpid()}"
        run([_nvcc(), "-shared", "-o", tmp] + objects)
        os.replace(tmp, LIB)
    build_native(run, headers, force)
    return LIB


def build_native(run, headers, force: bool) -> None:
    import sysconfig
    try:
        import torch
    except ImportError:
        sys.stderr.write("no torch: _kv_native.so is not built\n")
        return
    src = os.path.join(CSRC, "kv_binding.cpp")
    # a module of another torch or Python does not load, or worse: which ones it was built for is kept beside the objects
    built_for, stamp = f"{torch.__version__} {torch.__file__} {sysconfig.get_config_var('SOABI')}", os.path.join(OBJ_DIR, "_kv_native.built_for")
    same = os.path.exists(stamp) and open(stamp).read() == built_for
    if not force and same and os.path.exists(NATIVE) and os.path.getmtime(NATIVE) >= max(os.path.getmtime(p) for p in headers + [src]):
        return
    t = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    tmp = NATIVE + f".tmp{os.getpid()}"
    run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
         "-I" + INCLUDE, f"-I{t}/include", f"-I{t}/include/torch/csrc/api/include", f"-I{cuda}/include",
         "-I" + sysconfig.get_paths()["include"], src, "-o", tmp, f"-L{PKG}", "-l:liblexi_moe.so", "-Wl,-rpath,$ORIGIN",
         f"-L{t}/lib", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", f"-Wl,-rpath,{t}/lib"])
    os.replace(tmp, NATIVE)
    with open(stamp, "w") as f:
        f.write(built_for)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
