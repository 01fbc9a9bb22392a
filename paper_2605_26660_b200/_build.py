"""In-tree build of the CUDA library (nvcc, sm_100a only) and of the compiled part of its Python binding (g++)."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libwindq.so")
STAMP = LIB + ".srchash"
BINDING = os.path.join(HERE, "_binding.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--fmad=false",            # no contraction beyond the fma's written in the source
    "-Xcompiler", "-fPIC", "-shared", "--threads", "0",
]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def source_hash() -> str:
    h = hashlib.sha256()
    files = sources() + sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh"))
    files.append(os.path.join(INCLUDE, "windq.h"))
    for f in files:
        h.update(os.path.basename(f).encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def is_current() -> bool:
    if not (os.path.exists(LIB) and os.path.exists(STAMP)):
        return False
    with open(STAMP) as fh:
        return fh.read().strip() == source_hash()


def nvcc_path() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the windq CUDA library cannot be built")


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and is_current():
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc_path(), *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, "-o", tmp, *sources()]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    with open(STAMP, "w") as fh:
        fh.write(source_hash())
    return LIB


# ---- the compiled binding: csrc/binding.cpp against torch's headers, linked to the library beside it ----

BINDING_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden"]


def binding_command(out: str):
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    include = os.path.join(base, "include")
    return [shutil.which("g++") or "g++", *BINDING_FLAGS, "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
            "-I", INCLUDE, "-I", include, "-I", os.path.join(include, "torch", "csrc", "api", "include"),
            "-I", os.path.join(os.path.dirname(os.path.dirname(nvcc_path())), "include"), "-I", sysconfig.get_paths()["include"],
            os.path.join(CSRC, "binding.cpp"), "-o", out, "-L", HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN",
            "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]


def binding_hash() -> str:
    """Of all that a built binding fits: its sources, this Python and this torch.  Needs no compiler."""
    import sys

    import torch
    h = hashlib.sha256(" ".join([torch.__version__, str(torch._C._GLIBCXX_USE_CXX11_ABI), sys.version, *BINDING_FLAGS]).encode())
    for f in (os.path.join(CSRC, "binding.cpp"), os.path.join(INCLUDE, "windq.h")):
        with open(f, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def build_binding(force: bool = False) -> str:
    """Builds _binding.so unless it is current.  The library has to be there."""
    stamp = BINDING + ".srchash"
    if not force and os.path.exists(BINDING) and os.path.exists(stamp):
        with open(stamp) as fh:
            if fh.read().strip() == binding_hash():
                return BINDING
    tmp = BINDING + ".tmp.%d" % os.getpid()
    subprocess.run(binding_command(tmp), check=True)
    os.replace(tmp, BINDING)
    with open(stamp, "w") as fh:
        fh.write(binding_hash())
    return BINDING


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build_binding(force=True))
