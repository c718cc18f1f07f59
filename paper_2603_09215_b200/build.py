"""Compile the CUDA library (sm_100a) and the torch marshalling of its paged calls in-tree: ``python -m paper_2603_09215_b200.build``."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparsk.so")
PAGED = os.path.join(HERE, "_paged.so")
SOURCES = ["sparsk_api.cu", "sparsk_ops.cu", "sparsk_noalloc.cu", "sparsk_paged.cu", "sparsk_paged_attn.cu"]


def _stale() -> bool:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "sparsk.h"))
    return any(not os.path.exists(so) or os.path.getmtime(p) > os.path.getmtime(so) for so in (LIB, PAGED) for p in deps)


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
    side = _paged_command()
    with subprocess.Popen(side) as p:  # beside the CUDA sources
        subprocess.run(cmd, check=True)
    if p.returncode:
        raise subprocess.CalledProcessError(p.returncode, side)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
