"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension)."""
from __future__ import annotations

import os
import re
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libopt_tree.so")
OBJECTS = os.path.join(_HERE, "_build")
# Each source with its own flags (the tree kernels are all held to 80 registers, the cache kernels state theirs themselves).
SOURCES = [("opt_tree.cu", ["-maxrregcount=80"]), ("kv.cu", [])]
NVCC = "/usr/local/cuda/bin/nvcc"
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
NVCC_FLAGS = ARCH + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]


def _older(target: str, deps) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def dependencies(path: str) -> set:
    """A source and the headers that it includes by name, and those that they include."""
    found, todo = set(), [os.path.normpath(path)]
    while todo:
        at = todo.pop()
        if at in found or not os.path.exists(at):
            continue
        found.add(at)
        with open(at) as f:
            todo += [os.path.normpath(os.path.join(os.path.dirname(at), name)) for name in re.findall(r'^\s*#\s*include\s*"([^"]+)"', f.read(), re.M)]
    return found


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles what is older than its sources, the sources side by side, and links."""
    api = os.path.join(_HERE, "..", "include", "opt_tree.h")
    everything = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [api, os.path.abspath(__file__)]
    if not force and not _older(LIB, everything):
        return LIB
    os.makedirs(OBJECTS, exist_ok=True)
    objects, jobs = [], []
    for name, flags in SOURCES:
        src, obj = os.path.join(CSRC, name), os.path.join(OBJECTS, name + ".o")
        objects.append(obj)
        if force or _older(obj, dependencies(src) | {os.path.abspath(__file__)}):
            new = f"{obj}.{os.getpid()}.o"
            cmd = [NVCC] + NVCC_FLAGS + flags + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", new, src]
            jobs.append((subprocess.Popen(cmd), cmd, new, obj))
    for proc, cmd, new, obj in jobs:
        if proc.wait() != 0:
            for other, *_ in jobs:
                other.wait()
            raise subprocess.CalledProcessError(proc.returncode, cmd)
        os.replace(new, obj)
    new = f"{LIB}.{os.getpid()}.so"
    subprocess.check_call([NVCC] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-o", new] + objects)
    os.replace(new, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
