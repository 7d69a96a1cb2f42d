"""Build librelation.so (the CUDA kernels + C ABI) in-tree for sm_103a.

Each ``csrc/*.cu`` file is compiled to an object in parallel with
``nvcc -gencode arch=compute_103a,code=sm_103a -O3 -lineinfo``, then the objects are
linked into ``paper_2608_20172_gb300/_build/librelation.so`` with the static CUDA
runtime.  Beside it ``csrc/torch_calls.cpp``, the serving calls of the Python binding in native
code, becomes ``_build/relation_calls.so`` (host code against torch's headers; where these are
not installed the binding does the same in Python).  The driver API entry point used for TMA descriptors is resolved at run
time through the runtime, so the library loads on machines without a GPU driver.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import hashlib
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "librelation.so")
CALLS = os.path.join(BUILD, "relation_calls.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
              "--expt-relaxed-constexpr", f"-I{INCLUDE}", f"-I{CSRC}"]
CALLS_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-shared"]


def _nvcc() -> str:
    home = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cand = os.path.join(home, "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps_digest() -> str:
    h = hashlib.sha256()
    files = _sources() + sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + \
        sorted(glob.glob(os.path.join(CSRC, "*.h"))) + [os.path.join(INCLUDE, "relation.h")]
    for f in files:
        h.update(f.encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(ARCH + NVCC_FLAGS).encode())
    return h.hexdigest()


def _calls_digest(torch) -> str:
    """Of what relation_calls.so is made from and for: its sources, this torch and this Python."""
    h = hashlib.sha256()
    for f in (os.path.join(CSRC, "torch_calls.cpp"), os.path.join(INCLUDE, "relation.h")):
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(f"{torch.__version__} {torch._C._GLIBCXX_USE_CXX11_ABI} {sys.version} "
             f"{CALLS_FLAGS}".encode())
    return h.hexdigest()


def calls_current(path: str) -> bool:
    """Whether the relation_calls.so at path was built from these sources for this torch."""
    import torch

    try:
        with open(path + ".stamp") as f:
            return os.path.exists(path) and f.read().strip() == _calls_digest(torch)
    except OSError:
        return False


def _calls_not_built(why) -> None:
    """Say so, and leave no file of an earlier build: it is not that of these sources."""
    print(f"relation_calls.so not built: {why}", file=sys.stderr)
    for f in (CALLS + ".stamp", CALLS):
        if os.path.exists(f):
            os.remove(f)


def build_calls(force: bool = False) -> str | None:
    """Compile relation_calls.so; returns its path, None where it cannot be built."""
    try:
        import torch
    except ImportError as e:
        return _calls_not_built(e)

    if not force and calls_current(CALLS):
        return CALLS
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda"
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = ["g++", *CALLS_FLAGS,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f"-I{root}/include", f"-I{root}/include/torch/csrc/api/include",
           f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}/include", f"-I{INCLUDE}",
           os.path.join(CSRC, "torch_calls.cpp"),
           f"-L{root}/lib", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-o", tmp]
    digest = _calls_digest(torch)
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        return _calls_not_built(e)
    if r.returncode != 0:
        return _calls_not_built(f"\n{r.stderr}")
    os.replace(tmp, CALLS)
    with open(CALLS + ".stamp", "w") as f:
        f.write(digest)
    return CALLS


def build(force: bool = False, verbose: bool = False, extra_flags=None) -> str:
    """Compile and link librelation.so; returns its path.  Skips work when the
    sources are unchanged since the last build."""
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=1) as beside:
        calls = beside.submit(build_calls, force)
        lib = _build_lib(force, verbose, extra_flags)
        calls.result()
    return lib


def _build_lib(force, verbose, extra_flags) -> str:
    stamp = os.path.join(BUILD, "librelation.stamp")
    digest = _deps_digest() + (" ".join(extra_flags) if extra_flags else "")
    if not force and os.path.exists(LIB) and os.path.exists(stamp):
        if open(stamp).read().strip() == digest:
            return LIB
    nvcc = _nvcc()
    flags = ARCH + NVCC_FLAGS + list(extra_flags or [])

    headers = sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + \
        sorted(glob.glob(os.path.join(CSRC, "*.h"))) + [os.path.join(INCLUDE, "relation.h")]

    def obj_digest(src):
        h = hashlib.sha256()
        for f in [src] + headers:
            with open(f, "rb") as fh:
                h.update(fh.read())
        h.update(" ".join(flags).encode())
        return h.hexdigest()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        ostamp = obj + ".stamp"
        dig = obj_digest(src)
        if not force and os.path.exists(obj) and os.path.exists(ostamp) and \
                open(ostamp).read().strip() == dig:
            return obj
        cmd = [nvcc] + flags + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr, flush=True)
        with open(ostamp, "w") as f:
            f.write(dig)
        return obj

    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc] + ARCH + ["-shared", "-cudart", "static", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    with open(stamp, "w") as f:
        f.write(digest)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose=True))
