"""Builds libthanos.so (sm_100a) in-tree with nvcc.  No torch extension machinery: the library
has a plain C ABI and is loaded with ctypes.  Beside it _calls.so, with g++ against torch's headers:
the short way from Python to the entry points whose calls are as long as their kernels.  The library does
not need it: where g++ or torch's headers are missing, it is left out with a warning."""

from __future__ import annotations

import hashlib
import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libthanos.so")
CALLS = os.path.join(HERE, "_calls.so")
BUILD = os.path.join(HERE, "_build")
STAMP = os.path.join(BUILD, "stamp.txt")
CALLS_STAMP = os.path.join(BUILD, "calls_stamp.txt")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xptxas=-v",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-O3", "-I", INCLUDE, "-I", CSRC,
]


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _digest():
    h = hashlib.sha256()
    names = [f for f in sorted(os.listdir(CSRC)) if not f.endswith(".cpp")]
    for f in names + ["../../include/thanos.h"]:
        p = os.path.join(CSRC, f)
        if os.path.isfile(p):
            h.update(f.encode())
            h.update(open(p, "rb").read())
    # flags, not folders: a built tree may be moved
    h.update(" ".join(f for f in NVCC_FLAGS if f not in (INCLUDE, CSRC)).encode())
    return h.hexdigest()


def _torch():
    """Folder and version of the installed torch, without importing it."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("torch is not installed")
    root = os.path.dirname(spec.origin)
    text = open(os.path.join(root, "version.py")).read()
    return root, re.search(r"^__version__ = '(.+)'", text, re.M).group(1)


CALLS_SOURCE = os.path.join(CSRC, "calls.cpp")
CALLS_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-shared"]
CALLS_LIBS = ["-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]


def _calls_digest():
    h = hashlib.sha256(" ".join(CALLS_FLAGS + CALLS_LIBS + [sys.version, _torch()[1]]).encode())
    for f in (CALLS_SOURCE, os.path.join(INCLUDE, "thanos.h")):
        h.update(open(f, "rb").read())
    return h.hexdigest()


def _calls_command(out):
    torch, version = _torch()
    cuda = os.path.dirname(os.path.dirname(nvcc_path()))
    include = [os.path.join(torch, "include"),
               os.path.join(torch, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include"), INCLUDE]
    built_for = '-DTHANOS_BUILT_FOR="torch %s, python %d.%d"' % ((version,) + sys.version_info[:2])
    return (["g++"] + CALLS_FLAGS + [built_for, CALLS_SOURCE, "-o", out] + ["-I" + i for i in include]
            + ["-L" + os.path.join(torch, "lib")] + CALLS_LIBS)


class _Calls:
    """_calls.so on its way: compiled while the library is, put in its place when it is complete."""

    def __init__(self, force: bool):
        self.new = os.path.join(BUILD, "_calls.%d.so" % os.getpid())
        self.run = self.error = None
        try:
            self.digest = _calls_digest()
            if not force and os.path.exists(CALLS) and os.path.exists(CALLS_STAMP) \
                    and open(CALLS_STAMP).read().strip() == self.digest:
                return
            self.run = subprocess.Popen(_calls_command(self.new), stdout=subprocess.PIPE,
                                        stderr=subprocess.STDOUT, text=True)
        except Exception as e:   # no compiler, no torch, torch without its headers
            self.error = str(e)

    def finish(self):
        if self.run is not None:
            out, _ = self.run.communicate()
            if self.run.returncode != 0:
                self.error = "g++ failed\n" + out[-2000:]
        if self.error is not None:
            # one that is there may be of other sources
            for f in (CALLS, self.new):
                if os.path.exists(f):
                    os.remove(f)
            sys.stderr.write("warning: %s is not built, calls from Python take the long way: %s\n"
                             % (os.path.basename(CALLS), self.error))
        elif self.run is not None:
            os.replace(self.new, CALLS)   # not written over: a process may have it mapped
            open(CALLS_STAMP, "w").write(self.digest)


def nvcc_path():
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; the CUDA library cannot be built")


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into libthanos.so, and calls.cpp into _calls.so, unless they are
    already up to date."""
    os.makedirs(BUILD, exist_ok=True)
    calls = _Calls(force)
    try:
        return _build_library(force, verbose)
    finally:
        calls.finish()


def _build_library(force: bool, verbose: bool) -> str:
    dig = _digest()
    if not force and os.path.exists(LIB) and os.path.exists(STAMP):
        if open(STAMP).read().strip() == dig:
            return LIB
    nvcc = nvcc_path()
    objs = []
    procs = []
    for src in _sources():
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
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
    open(os.path.join(BUILD, "ptxas.log"), "w").write("\n".join(log))
    if failed:
        sys.stderr.write("\n".join(log))
        raise RuntimeError("nvcc failed")
    if verbose:
        print("\n".join(log))
    cmd = [nvcc, "-shared", "-o", LIB] + objs + ["-lcudart"]
    subprocess.run(cmd, check=True)
    open(STAMP, "w").write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
