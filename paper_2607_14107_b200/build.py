"""Build the C-ABI shared library (libpolestar.so) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
import time
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "obj")                            # object files and their dependency lists
UNITS = ["polestar", "operators"]                          # translation units, compiled side by side
OUT = os.path.join(HERE, "libpolestar.so")
OUT_TRACE = os.path.join(HERE, "libpolestar_trace.so")     # same library with kernel time stamps compiled in


def _deps():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    files.append(os.path.join(os.path.dirname(HERE), "include", "polestar.h"))
    return files


def needs_build(out: str = OUT) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(f) > t for f in _deps())


def _unit_is_current(obj: str, dep: str) -> bool:
    """Whether an object is newer than every file of this tree that it was compiled from."""
    if not (os.path.exists(obj) and os.path.exists(dep)):
        return False
    with open(dep) as f:
        files = f.read().replace("\\\n", " ").split()[1:]
    root, t = os.path.dirname(HERE), os.path.getmtime(obj)
    own = [p for p in (os.path.abspath(p) for p in files if p != ":") if p.startswith(root + os.sep)]
    return len(own) > 0 and all(os.path.exists(p) and os.path.getmtime(p) <= t for p in own)


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("nvcc failed building libpolestar.so")
    return r.stderr


def build(force: bool = False, verbose: bool = False, trace: bool = False) -> str:
    """Compile libpolestar.so (or, with ``trace``, libpolestar_trace.so: -DPOLESTAR_TRACE adds the
    per-kernel time stamps that `timeline.py` reads; select it with POLESTAR_LIB)."""
    out = OUT_TRACE if trace else OUT
    if not force and not needs_build(out):
        return out
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    os.makedirs(OBJ, exist_ok=True)
    started = time.time()                                  # outputs carry this time: a file edited during the build is newer than they are

    def compile_unit(name: str) -> str:
        stem = os.path.join(OBJ, name + ("_trace" if trace else ""))
        if not force and _unit_is_current(stem + ".o", stem + ".d"):
            return ""
        cmd = [nvcc, "-c", "-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo", *arch, "-MD", "-MF", stem + ".d",
               os.path.join(CSRC, name + ".cu"), "-o", stem + ".o"]
        if trace:
            cmd.insert(1, "-DPOLESTAR_TRACE")
        if verbose:
            cmd[1:1] = ["-Xptxas", "-v"]
        said = _run(cmd)
        os.utime(stem + ".o", (started, started))
        return said

    with ThreadPoolExecutor(len(UNITS)) as pool:
        said = list(pool.map(compile_unit, UNITS))
    if verbose:
        sys.stderr.write("".join(said))
    _run([nvcc, "-shared", *arch, *[os.path.join(OBJ, n + ("_trace" if trace else "") + ".o") for n in UNITS], "-o", out])
    os.utime(out, (started, started))
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, trace="--trace" in sys.argv))
