"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import hashlib
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB_DIR = PKG / "lib"
OBJ_DIR = LIB_DIR / "obj"
LIB = LIB_DIR / "libesc_convattn.so"
INCLUDE = PKG.parent / "include"

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the ConvAttn CUDA library cannot be built")


def sources():
    return sorted(CSRC.glob("*.cu"))


def _includes(path: Path, seen: set) -> set:
    """`path` and the files of this package that it includes, directly or not."""
    if path in seen or not path.exists():
        return seen
    seen.add(path)
    for name in re.findall(r'^\s*#include "([^"]+)"', path.read_text(), flags=re.M):
        _includes((path.parent / name).resolve(), seen)
    return seen


def _newest(src: Path) -> float:
    return max(p.stat().st_mtime for p in _includes(src.resolve(), set()))


def _object(src: Path) -> Path:
    """Its object file: another one where the compiler is given other flags."""
    return OBJ_DIR / f"{src.stem}.{hashlib.sha256(' '.join(NVCC_FLAGS).encode()).hexdigest()[:8]}.o"


def _left_over() -> list:
    """Object files of other flags, or of sources that are gone."""
    return [o for o in OBJ_DIR.glob("*.o") if ".tmp" not in o.name and o not in {_object(s) for s in sources()}]


def needs_build() -> bool:
    if not LIB.exists() or _left_over():
        return True
    t = LIB.stat().st_mtime
    deps = list(CSRC.glob("*.cu")) + list(CSRC.glob("*.cuh")) + list(CSRC.glob("*.h")) + list(INCLUDE.glob("*.h"))
    return any(d.stat().st_mtime > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every .cu under csrc/ (side by side) and link lib/libesc_convattn.so.

    Without `force` an object file of these flags, newer than its source and everything that one includes, is taken as it is;
    `verbose` prints the registers of what is compiled."""
    if not force and not needs_build():
        return LIB
    LIB_DIR.mkdir(exist_ok=True)
    OBJ_DIR.mkdir(exist_ok=True)
    flags = [*NVCC_FLAGS, *(["-Xptxas=-v"] if verbose else []), "-I", str(INCLUDE)]

    def compiled(src: Path) -> Path:
        obj = _object(src)
        if force or not obj.exists() or obj.stat().st_mtime <= _newest(src):
            tmp = obj.with_suffix(".tmp%d.o" % os.getpid())
            subprocess.check_call([_nvcc(), *flags, "-c", "-o", str(tmp), str(src)])
            os.replace(tmp, obj)
        return obj

    with ThreadPoolExecutor() as pool:
        objects = list(pool.map(compiled, sources()))
    tmp = LIB.with_suffix(".so.tmp%d" % os.getpid())
    subprocess.check_call([_nvcc(), *NVCC_FLAGS, "-shared", "-o", str(tmp), *map(str, objects)])
    os.replace(tmp, LIB)
    for old in _left_over():
        old.unlink(missing_ok=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
