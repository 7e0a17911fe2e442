"""Build libparason.so (CUDA kernels for sm_103a + host planner) in-tree.

Every translation unit compiles in parallel with nvcc (sm_103a only) or g++,
then nvcc links one shared library into paper_2608_24658_gb300/_build/.
No cmake, no torch extension machinery: the library has a plain C ABI.  Beside it
stands a small module of the Python binding, csrc/python/tensors.cpp, which reads torch's
tensors: built for one torch and one Python, whose versions are in its name.  The library
needs neither: where torch, Python's headers or torch's C++ ones are missing, or do not
compile, there is no module, and the binding's own checks serve.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libparason.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
TENSORS_SRC = os.path.join(CSRC, "python", "tensors.cpp")


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


def _tensors():
    """The path of the binding's module, or None where there is nothing to build it with."""
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return None
    try:
        import torch
    except ImportError:
        return None
    return os.path.join(BUILD, f"_tensors-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def _build_tensors(path: str) -> str:
    """The binding's module; where it does not compile, a note of that in its place."""
    import torch
    torch_home, include = os.path.dirname(torch.__file__), sysconfig.get_paths()["include"]
    tmp = path + f".tmp{os.getpid()}"
    lib = os.path.join(torch_home, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-isystem", os.path.join(torch_home, "include"),
           "-I", include, f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", TENSORS_SRC, "-o", tmp,
           "-L", lib, f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode == 0:
        os.replace(tmp, path)
        return res.stderr
    if os.path.exists(path):
        os.remove(path)
    with open(_failed(path), "w") as f:
        f.write(f"{' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    sys.stderr.write(f"the binding's module did not compile, and tensors are looked at without it; see {_failed(path)}\n")
    return ""


def _failed(path: str) -> str:
    return path + ".failed"


def _newer(path: str, sources) -> bool:
    return os.path.exists(path) and os.path.getmtime(path) >= max(map(os.path.getmtime, sources))


def build(force: bool = False, verbose_ptxas: bool = False, quiet: bool = True) -> str:
    """Compile and link libparason.so, and the binding's module, if any source or header is
    newer than they are."""
    srcs, headers = _sources()
    force = force or verbose_ptxas
    stale = force or not _newer(LIB, srcs + headers + [__file__])
    module = _tensors()
    if module and not force and any(_newer(p, [__file__, TENSORS_SRC]) for p in (module, _failed(module))):
        module = None
    if not stale and module is None:
        return LIB
    cuda = _cuda_home()
    os.makedirs(BUILD, exist_ok=True)
    objs = [os.path.join(BUILD, os.path.basename(s) + ".o") for s in srcs]
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        futs = {ex.submit(_compile, s, o, cuda, verbose_ptxas): s for s, o in zip(srcs, objs)} if stale else {}
        if module:
            futs[ex.submit(_build_tensors, module)] = TENSORS_SRC
        for f in cf.as_completed(futs):
            log = f.result()
            if log and (verbose_ptxas or not quiet):
                sys.stderr.write(f"== {os.path.basename(futs[f])}\n{log}")
    if not stale:
        return LIB
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
