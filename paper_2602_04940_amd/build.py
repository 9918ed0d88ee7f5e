"""Compile the gfx950 HIP library ``libts3.so`` and the binding's tensor-table module
``_tensors.so`` in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(PKG, "csrc", "ts3.hip")
LIB = os.path.join(PKG, "libts3.so")
TENSORS_SRC = os.path.join(PKG, "csrc", "tensors.cpp")
TENSORS = os.path.join(PKG, "_tensors.so")

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # Packed fp32 instructions are kept out of the generated code.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libts3.so)")


def tensors_command(out: str) -> list[str]:
    """Host code against this Python and this torch: their headers, and torch's libraries by path."""
    import torch
    from torch.utils import cpp_extension
    gxx = shutil.which("g++")
    if not gxx:
        raise RuntimeError("g++ not found")
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = [sysconfig.get_paths()["include"], *cpp_extension.include_paths()]
    return [gxx, "-O2", "-std=c++17", "-fPIC", "-shared",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *["-I" + p for p in include], "-o", out,
            TENSORS_SRC, "-L" + libs, "-Wl,-rpath," + libs, "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(cmd, job, verbose):
    """Waits for a compiler; raises with its output if it failed."""
    out = job.communicate()[0]
    msgs = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
    if job.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed ({job.returncode}):\n{' '.join(cmd)}\n{msgs}")
    if verbose and msgs.strip():
        print(msgs)


def build_library(verbose: bool = False) -> str:
    """Always recompiles both, side by side; writes to temporary names and renames on success.  The
    library needs hipcc alone.  Where the tensor-table module, which GradClip reads its lists with,
    cannot be built, an older one is removed and a warning says so: the rest works without it."""
    tmp, tensors_tmp = LIB + ".tmp", TENSORS + ".tmp"
    cmd = [hipcc(), *HIP_FLAGS, "-o", tmp, SRC]
    job = _start(cmd)
    try:
        tensors_cmd = tensors_command(tensors_tmp)
        _finish(tensors_cmd, _start(tensors_cmd), verbose)
        os.replace(tensors_tmp, TENSORS)
    except Exception as e:
        if os.path.exists(TENSORS):
            os.remove(TENSORS)
        warnings.warn(f"{os.path.basename(TENSORS)} could not be built, GradClip will not work: {e}")
    finally:
        _finish(cmd, job, verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
