"""Compile the CUDA library (sm_100a) and the torch marshalling of its paged calls in-tree: ``python -m paper_2603_09215_b200.build``.

The library needs nvcc alone, and is built whatever becomes of the marshalling: callers of the C ABI have no use for that.  Without torch it
is left out; where torch is there and it does not compile, that is an error, raised when the library is in its place."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparsk.so")
PAGED = os.path.join(HERE, "_paged.so")
SOURCES = ["sparsk_api.cu", "sparsk_ops.cu", "sparsk_noalloc.cu", "sparsk_paged.cu", "sparsk_paged_attn.cu"]


def _have_torch() -> bool:
    return importlib.util.find_spec("torch") is not None


def _stale() -> bool:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "sparsk.h"))
    made = (LIB, PAGED) if _have_torch() else (LIB,)
    return any(not os.path.exists(so) or os.path.getmtime(p) > os.path.getmtime(so) for so in made for p in deps)


def _paged_command() -> list[str]:
    import torch
    at = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in (os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
              sysconfig.get_paths()["include"], os.path.join(cuda, "include")):
        cmd += ["-isystem", d]
    return cmd + ["-o", PAGED, os.path.join(CSRC, "sparsk_torch.cpp"), "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu",
                  "-lc10", "-lc10_cuda"]


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    cmd = ["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "--use_fast_math", "--threads", "0", "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    cmd += ["-lcuda"]
    with subprocess.Popen(cmd) as lib:
        problem = _build_paged()  # beside the CUDA sources
    if lib.returncode:
        raise subprocess.CalledProcessError(lib.returncode, cmd)
    if problem:
        raise RuntimeError(f"{LIB} is built, but {PAGED}, which the Python binding's paged calls need, is not: {problem}")
    return LIB


def _build_paged() -> str | None:
    """What went wrong, if something did."""
    if not _have_torch():
        print(f"no torch here: {PAGED}, which only the Python binding needs, is left out", file=sys.stderr)
        return None
    try:
        subprocess.run(_paged_command(), check=True)
    except Exception as e:  # (an import of torch that fails can raise anything)
        return str(e)
    return None


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
