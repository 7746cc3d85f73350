"""Builds libthanos.so (sm_100a) in-tree with nvcc.  No torch extension machinery: the library
has a plain C ABI and is loaded with ctypes.  Beside it _calls.so, with g++ against torch's headers:
the short way from Python to the entry points whose calls are as long as their kernels."""

from __future__ import annotations

import hashlib
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libthanos.so")
CALLS = os.path.join(HERE, "_calls.so")
STAMP = os.path.join(HERE, "_build", "stamp.txt")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xptxas=-v",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-O3", "-I", INCLUDE, "-I", CSRC,
]


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _digest():
    h = hashlib.sha256()
    names = sorted(os.listdir(CSRC)) + ["../../include/thanos.h"]
    for f in names:
        p = os.path.join(CSRC, f)
        if os.path.isfile(p):
            h.update(f.encode())
            h.update(open(p, "rb").read())
    # flags, not folders: a built tree may be moved
    h.update(" ".join(f for f in NVCC_FLAGS if f not in (INCLUDE, CSRC)).encode())
    h.update((sys.version + importlib.metadata.version("torch")).encode())
    return h.hexdigest()


def _calls_command():
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.dirname(os.path.dirname(nvcc_path()))
    include = [os.path.join(torch, "include"),
               os.path.join(torch, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include"), INCLUDE]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", os.path.join(CSRC, "calls.cpp"), "-o",
             CALLS] + ["-I" + i for i in include] + ["-L" + os.path.join(torch, "lib")]
            + ["-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"])


def nvcc_path():
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; the CUDA library cannot be built")


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into libthanos.so unless it is already up to date."""
    dig = _digest()
    if not force and os.path.exists(LIB) and os.path.exists(CALLS) and os.path.exists(STAMP):
        if open(STAMP).read().strip() == dig:
            return LIB
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    nvcc = nvcc_path()
    objs = []
    procs = [("calls.cpp", subprocess.Popen(_calls_command(), stdout=subprocess.PIPE,
                                            stderr=subprocess.STDOUT, text=True))]
    for src in _sources():
        obj = os.path.join(bdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc] + NVCC_FLAGS + ["-c", src, "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    log = []
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        log.append("== %s\n%s" % (os.path.basename(src), out))
        failed |= p.returncode != 0
    open(os.path.join(bdir, "ptxas.log"), "w").write("\n".join(log))
    if failed:
        sys.stderr.write("\n".join(log))
        raise RuntimeError("nvcc or g++ failed")
    if verbose:
        print("\n".join(log))
    cmd = [nvcc, "-shared", "-o", LIB] + objs + ["-lcudart"]
    subprocess.run(cmd, check=True)
    open(STAMP, "w").write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
