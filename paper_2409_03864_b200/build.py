"""Build the CUDA library in-tree: csrc/*.cu -> libtdx.so (sm_100a only)."""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libtdx.so"

OBJ = PKG / "build"

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC",
    "-Xptxas", "-v",
]


def sources():
    return sorted(CSRC.glob("*.cu"))


def _includes(path: Path, seen: set) -> set:
    """The file and what it includes of this repository."""
    if path not in seen:
        seen.add(path)
        for name in re.findall(r'^#include "([^"]+)"', path.read_text(), re.M):
            for folder in (CSRC, ROOT / "include"):
                if (folder / name).exists():
                    _includes(folder / name, seen)
    return seen


def _newer(target: Path, files) -> bool:
    """Whether one of the files was changed after the target was made (or there is no target)."""
    return not target.exists() or any(f.stat().st_mtime > target.stat().st_mtime for f in files)


def _stale() -> bool:
    return any(_newer(LIB, _includes(s, set())) for s in sources())


def _run(cmd, verbose):
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
    if proc.returncode != 0:
        raise RuntimeError(f"nvcc failed building {cmd[cmd.index('-o') + 1]}")


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile with nvcc (cross-compiles without a GPU), one object per source, side by side.  Returns the path of libtdx.so."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    OBJ.mkdir(exist_ok=True)
    tag = f".tmp{os.getpid()}"
    objects = {s: OBJ / (s.stem + ".o") for s in sources()}
    todo = [s for s, o in objects.items() if force or _newer(o, _includes(s, set()))]

    def compile_one(source):
        out = objects[source]
        tmp = out.with_name(out.name + tag)
        _run([nvcc, *NVCC_FLAGS, "-I", str(ROOT / "include"), "-I", str(CSRC), "-c", "-o", str(tmp), str(source)], verbose)
        os.replace(tmp, out)

    with ThreadPoolExecutor() as pool:
        list(pool.map(compile_one, todo))
    tmp = LIB.with_suffix(".so" + tag)
    _run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", str(tmp)] + [str(o) for o in objects.values()], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True)
    print(LIB)
