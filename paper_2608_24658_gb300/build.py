"""Build libparason.so (CUDA kernels for sm_103a + host planner) in-tree.

Every translation unit compiles in parallel with nvcc (sm_103a only) or g++,
then nvcc links one shared library into paper_2608_24658_gb300/_build/.
No cmake, no torch extension machinery: the library has a plain C ABI.  Beside it
stands a small module of the Python binding, csrc/python/tensors.cpp, which reads torch's
tensors: built for one torch and one Python, whose versions are in its name.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libparason.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
TENSORS_SRC = os.path.join(CSRC, "python", "tensors.cpp")
TENSORS = os.path.join(BUILD, f"_tensors-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def _cuda_home() -> str:
    env = os.environ.get("CUDA_HOME") or os.environ.get("CUDA_PATH")
    if env and os.path.isdir(env):
        return env
    nvcc = shutil.which("nvcc")
    if nvcc:
        return os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
    return "/usr/local/cuda"


def _sources():
    srcs = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cpp")))
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(INCLUDE, "parason.h"))
    return [os.path.join(CSRC, s) for s in srcs], headers


def _compile(src: str, obj: str, cuda: str, verbose_ptxas: bool) -> str:
    nvcc = os.path.join(cuda, "bin", "nvcc")
    inc = ["-I", INCLUDE, "-I", CSRC, "-I", os.path.join(cuda, "include")]
    if src.endswith(".cu"):
        cmd = [nvcc, *ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
               "-Xcompiler", "-Wall", "--expt-relaxed-constexpr", *inc, "-c", src, "-o", obj]
        if verbose_ptxas:
            cmd.insert(1, "-Xptxas=-v")
    else:
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-Wextra", *inc, "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    return res.stderr


def _build_tensors() -> str:
    """The binding's module."""
    torch_home, include = os.path.dirname(torch.__file__), sysconfig.get_paths()["include"]
    tmp = TENSORS + f".tmp{os.getpid()}"
    lib = os.path.join(torch_home, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-isystem", os.path.join(torch_home, "include"),
           "-I", include, f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", TENSORS_SRC, "-o", tmp,
           "-L", lib, f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, TENSORS)
    return res.stderr


def build(force: bool = False, verbose_ptxas: bool = False, quiet: bool = True) -> str:
    """Compile and link libparason.so, and the binding's module, if any source or header is
    newer than they are."""
    srcs, headers = _sources()
    binding = os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))
    made = [LIB, TENSORS] if binding else [LIB]          # (without Python's headers: no module)
    if not force and not verbose_ptxas and all(map(os.path.exists, made)):
        newest = max(os.path.getmtime(p) for p in srcs + headers + [__file__, TENSORS_SRC])
        if min(map(os.path.getmtime, made)) >= newest:
            return LIB
    cuda = _cuda_home()
    os.makedirs(BUILD, exist_ok=True)
    objs = [os.path.join(BUILD, os.path.basename(s) + ".o") for s in srcs]
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        futs = {ex.submit(_compile, s, o, cuda, verbose_ptxas): s for s, o in zip(srcs, objs)}
        if binding:
            futs[ex.submit(_build_tensors)] = TENSORS_SRC
        for f in cf.as_completed(futs):
            log = f.result()
            if log and (verbose_ptxas or not quiet):
                sys.stderr.write(f"== {os.path.basename(futs[f])}\n{log}")
    tmp = LIB + f".tmp{os.getpid()}"
    nvcc = os.path.join(cuda, "bin", "nvcc")
    cmd = [nvcc, *ARCH, "-shared", "-Xcompiler", "-fPIC", "-o", tmp, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="--ptxas" in sys.argv, quiet=False))
