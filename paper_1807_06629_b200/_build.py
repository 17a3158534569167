"""Builds libprsgd.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB_PATH = os.path.join(HERE, "libprsgd.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC,
]


def _sources():
    out = [os.path.join(INCLUDE, "prsgd.h")]
    for f in sorted(os.listdir(CSRC)):
        if f.endswith((".cu", ".cuh", ".h")):
            out.append(os.path.join(CSRC, f))
    return out


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(s) > t for s in _sources())


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every csrc/*.cu (prsgd_api.cu includes the kernel headers of the training step, the others hold the
    stand-alone operators), one nvcc each side by side, and link them into libprsgd.so."""
    if not force and not is_stale():
        return LIB_PATH
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    units = [f for f in _sources() if f.endswith(".cu")]
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else [])
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(u) + ".o") for u in units]
        with ThreadPoolExecutor(len(units)) as pool:
            runs = list(pool.map(lambda uo: subprocess.run([nvcc] + flags + ["-c", uo[0], "-o", uo[1]], capture_output=True, text=True),
                                 zip(units, objs)))
        for res in runs:
            if res.returncode != 0:
                raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        link = subprocess.run([nvcc] + NVCC_FLAGS + ["-shared"] + objs + ["-o", LIB_PATH + ".tmp"], capture_output=True, text=True)
    if link.returncode != 0:
        raise RuntimeError("linking libprsgd.so failed:\n" + link.stdout + link.stderr)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    if verbose:
        for res in runs:
            print(res.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
