"""Builds libthinfer.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the torch marshalling module
_ops.so with the host compiler."""
from __future__ import annotations

import importlib.metadata
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libthinfer.so")            # IEEE FP16 storage
LIB_BF16 = os.path.join(HERE, "libthinfer_bf16.so")  # BF16 storage: the same sources with -DTHINFER_BF16
VARIANTS = ((LIB, []), (LIB_BF16, ["-DTHINFER_BF16"]))
OPS = os.path.join(HERE, "_ops.so")                  # Python module: torch tensors -> the C entry points
OPS_TORCH = OPS + ".torch"                           # the version of torch it was compiled for
OPS_SRC = os.path.join(CSRC, "torch_ops.cpp")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC",
    "--expt-relaxed-constexpr",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA extension cannot be built")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))) + [
        os.path.join(os.path.dirname(HERE), "include", "thinfer.h")]


def _torch_version():
    """Version of the installed torch (without importing it), None without one."""
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return None


def _ops_is_stale() -> bool:
    deps = (OPS_SRC, os.path.join(os.path.dirname(HERE), "include", "thinfer.h"))
    return not os.path.exists(OPS) or any(os.path.getmtime(s) > os.path.getmtime(OPS) for s in deps) or _ops_torch() != _torch_version()


def _ops_torch():
    """Version of torch that _ops.so was compiled for: it fits no other."""
    try:
        with open(OPS_TORCH) as f:
            return f.read().strip()
    except OSError:
        return None


def _ops_command():
    import torch
    root = os.path.dirname(torch.__file__)
    inc, lib = os.path.join(root, "include"), os.path.join(root, "lib")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-isystem", sysconfig.get_paths()["include"], "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"), "-isystem", cuda,
            OPS_SRC, "-o", OPS, "-L" + lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-Wl,-rpath," + lib]


def is_stale(lib: str = None) -> bool:
    libs = [lib] if lib else [v[0] for v in VARIANTS]
    if lib is None and _torch_version() is not None and _ops_is_stale():
        return True
    for l in libs:
        if not os.path.exists(l):
            return True
        t = os.path.getmtime(l)
        if any(os.path.getmtime(s) > t for s in sources()):
            return True
    return False


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu of csrc/ into one shared library per storage type and, where torch is installed, torch_ops.cpp
    into _ops.so (the compilations run side by side, and each leaves its result whatever becomes of the others); returns
    the path of the FP16 library."""
    cus = [s for s in sources() if s.endswith(".cu")]
    extra = os.environ.get("THINFER_NVCC_EXTRA", "").split()
    procs, failed = [], []
    for lib, defs in VARIANTS:
        if not force and not is_stale(lib):
            continue
        cmd = [_nvcc()] + NVCC_FLAGS + defs + extra + (["-Xptxas", "-v"] if verbose else []) + ["-o", lib] + cus
        procs.append((lib, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    if _torch_version() is not None and (force or _ops_is_stale()):   # without torch there is nothing to marshal
        try:
            procs.append((OPS, subprocess.Popen(_ops_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        except (OSError, ImportError) as e:                            # the libraries do not depend on it
            failed.append(f"the compiler cannot be run for {os.path.basename(OPS)}:\n{e}")
    for lib, p in procs:
        out, _ = p.communicate()
        if p.returncode == 0 and lib == OPS:
            with open(OPS_TORCH, "w") as f:
                f.write(_torch_version() + "\n")
        if p.returncode != 0:
            failed.append(f"the compiler failed for {os.path.basename(lib)}:\n" + out)
        elif verbose:
            print(out)
    if failed:
        raise RuntimeError("\n".join(failed))
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
