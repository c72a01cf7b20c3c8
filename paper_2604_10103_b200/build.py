"""Build libhf.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and libhf_host-<torch's version>.so, which looks over torch
tensors for the optimizer, with g++."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhf.so")
HOST_SOURCE = os.path.join(CSRC, "host_tensors.cpp")
HEADER = os.path.join(HERE, "..", "include", "hf.h")
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
]


def sources():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".cu")]


def _deps():
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))] + [HEADER]


def _older(lib, deps) -> bool:
    return not os.path.exists(lib) or any(os.path.getmtime(p) > os.path.getmtime(lib) for p in deps)


def host_lib() -> str:
    """Path of the host library for the torch that is installed: it is built against that one's inlined accessors.  ImportError without torch."""
    import torch
    return os.path.join(HERE, f"libhf_host-{torch.__version__}.so")


def _host_stale() -> bool:
    try:
        return _older(host_lib(), [HOST_SOURCE, HEADER])
    except ImportError:
        return False


def stale() -> bool:
    return _older(LIB, _deps()) or _host_stale()


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    return res.stderr


def _host_command():
    import torch
    root = os.path.dirname(torch.__file__)
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *("-I" + p for p in include), HOST_SOURCE, "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", host_lib()]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into libhf.so (returns its path), which needs no torch, and then, where torch is installed, host_tensors.cpp into its host
    library.  Raises on failure."""
    if force or _older(LIB, _deps()):
        nvcc = os.environ.get("NVCC", "nvcc")
        told = _run([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + sources() + ["-o", LIB])
        if verbose:
            sys.stderr.write(told)
    try:
        host = host_lib()
    except ImportError:
        sys.stderr.write("torch is not installed: built without the host library, which the optimizer's calls from Python need\n")
        return LIB
    if force or _older(host, [HOST_SOURCE, HEADER]):
        _run(_host_command())
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
