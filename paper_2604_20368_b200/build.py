"""Build the sm_100a shared library in-tree (nvcc cross-compiles without a GPU)."""
from __future__ import annotations

import contextlib
import glob
import os
import re
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_DIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIB_DIR, "liblaplace_nystrom.so")
OBJ_DIR = os.path.join(LIB_DIR, "obj")
ROOT = os.path.dirname(HERE)

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _depends(path: str, seen=None):
    """The file and every file it includes by a quoted path, directly or through another."""
    seen = set() if seen is None else seen
    path = os.path.normpath(path)
    if path not in seen and os.path.exists(path):
        seen.add(path)
        with open(path) as f:
            for inc in re.findall(r'^\s*#include\s+"([^"]+)"', f.read(), re.M):
                _depends(os.path.join(os.path.dirname(path), inc), seen)
    return seen


@contextlib.contextmanager
def _discarding(paths):
    """Those of the paths that still exist at the end are removed: what a compile that failed, or was interrupted, wrote."""
    try:
        yield
    finally:
        for p in paths:
            if os.path.exists(p):
                os.remove(p)


def _newest(paths) -> float:
    return max(os.path.getmtime(p) for p in paths)


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    return any(_newest(_depends(s)) > os.path.getmtime(LIB) for s in sources())


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu (side by side, each only if it or a file it includes changed) and link them into
    lib/liblaplace_nystrom.so."""
    if not (force or _stale()):
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    tag = f".tmp{os.getpid()}"
    objects = [os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o") for src in sources()]
    running = []
    with _discarding([p + tag for p in objects + [LIB]]):
        for src, obj in zip(sources(), objects):
            if force or not os.path.exists(obj) or _newest(_depends(src)) > os.path.getmtime(obj):
                cmd = ["nvcc"] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj + tag, src]
                running.append((subprocess.Popen(cmd), cmd, obj))
        failed = [cmd for proc, cmd, _ in running if proc.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        for _, _, obj in running:
            os.replace(obj + tag, obj)
        subprocess.check_call(["nvcc"] + NVCC_FLAGS + ["-shared", "-o", LIB + tag] + objects)
        os.replace(LIB + tag, LIB)
    return LIB


def marshal_path() -> str:
    """The Python module that marshals torch tensors.  It is linked against torch's C++ classes and Python's, so its name holds the
    versions that it was built for."""
    import torch
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    return os.path.join(LIB_DIR, f"_ln_torch.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}-abi{abi}.so")


def build_marshal(force: bool = False) -> str:
    """Compile csrc/ln_torch.cpp against torch's headers into marshal_path() if it or a file it includes changed."""
    import torch
    marshal = marshal_path()
    src = os.path.join(CSRC, "ln_torch.cpp")
    header = os.path.join(ROOT, "include", "laplace_nystrom.h")
    if not force and os.path.exists(marshal) and _newest([src, header]) <= os.path.getmtime(marshal):
        return marshal
    os.makedirs(LIB_DIR, exist_ok=True)
    torch_dir = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), os.path.join(torch_dir, "include"),
               os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
               os.path.join(cuda, "include")]
    lib = os.path.join(torch_dir, "lib")
    tmp = marshal + f".tmp{os.getpid()}"
    with _discarding([tmp]):
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-DTORCH_EXTENSION_NAME=_ln_torch",
                               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
                              + [f for d in include for f in ("-isystem" if d != include[0] else "-I", d)]
                              + [src, "-o", tmp, "-L" + lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
        os.replace(tmp, marshal)
    return marshal


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build_marshal(force=True))
