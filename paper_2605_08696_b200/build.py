"""Builds libsrm.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import hashlib
import os
import re
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libsrm.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xptxas=-v",
    "-Xcompiler", "-fPIC", "-cudart", "static",
]
UNITS = ["srm_api.cu", "ops8_api.cu"]      # translation units: the decode library; 8-bit operators and sampling per row
OBJ_DIR = os.path.join(PKG_DIR, "_build")


def _closure(unit):
    """A translation unit and every file of this repository that it includes."""
    todo, seen = [os.path.join(CSRC, unit)], []
    while todo:
        p = os.path.normpath(todo.pop())
        if p in seen:
            continue
        seen.append(p)
        with open(p) as f:
            todo += [os.path.join(os.path.dirname(p), i) for i in re.findall(r'^\s*#include "([^"]+)"', f.read(), re.M)]
    return sorted(seen)


def _unit_hash(unit) -> str:
    h = hashlib.sha256()
    for s in _closure(unit):
        with open(s, "rb") as f:
            h.update(f.read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def _source_hash() -> str:
    return "\n".join(f"{u} {_unit_hash(u)}" for u in UNITS)


def _read(path):
    if not os.path.exists(path):
        return None
    with open(path) as f:
        return f.read().strip()


def needs_build() -> bool:
    """True when libsrm.so is missing or was built from different sources."""
    return not os.path.exists(LIB_PATH) or _read(LIB_PATH + ".srchash") != _source_hash()


def _nvcc(args):
    return subprocess.run([shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"] + args, capture_output=True, text=True)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile the translation units of csrc/ (side by side; unchanged ones are kept) and link them into libsrm.so."""
    if not force and not needs_build():
        return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)

    def compile_unit(unit):
        obj = os.path.join(OBJ_DIR, unit + ".o")
        want = _unit_hash(unit)
        if not force and os.path.exists(obj) and _read(obj + ".srchash") == want:
            return obj, None
        res = _nvcc(NVCC_FLAGS + ["-c", "-o", obj, os.path.join(CSRC, unit)])
        if res.returncode == 0:
            with open(obj + ".ptxas", "w") as f:
                f.write(res.stderr)
            with open(obj + ".srchash", "w") as f:
                f.write(want)
        return obj, res

    with ThreadPoolExecutor(len(UNITS)) as pool:
        done = list(pool.map(compile_unit, UNITS))
    for (_, res), unit in zip(done, UNITS):
        if res is not None and (verbose or res.returncode != 0):
            sys.stderr.write(res.stdout + res.stderr)
        if res is not None and res.returncode != 0:
            raise RuntimeError(f"nvcc failed building {unit}")
    objs = [obj for obj, _ in done]
    res = _nvcc(NVCC_FLAGS[:2] + ["-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "-o", LIB_PATH] + objs)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed linking libsrm.so")
    with open(os.path.join(PKG_DIR, "ptxas_report.txt"), "w") as f:
        f.write("".join(_read(o + ".ptxas") + "\n" for o in objs))
    with open(LIB_PATH + ".srchash", "w") as f:
        f.write(_source_hash())
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
