"""Build the CUDA library in-tree: ``python -m paper_2602_02071_b200.build``.

Compiles the translation units of ``csrc/`` (``baps_lib.cu``: conversions, row softmax, BAPS attention; ``baps_serving.cu``:
windowed attention, the 8-bit key-value cache and its pages) for sm_100a, side by side, and links them into
``paper_2602_02071_b200/libbaps.so``.  nvcc cross-compiles, so no GPU is needed to build.  ``serving_marshal.cpp``, the binding's
argument checks of the serving calls, becomes the extension module ``_serving.so``.
"""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libbaps.so")
# Second build of the same sources for the wait test only: every bounded device-side wait gives up
# after 1 ms instead of 2 s, and the TMA producer can be told to leave one tile load out.  Nothing
# but tests/test_gpu_wait_timeout.py loads it.
WAIT_TEST_LIB = os.path.join(_HERE, "libbaps_waittest.so")
WAIT_TEST_FLAGS = ["-DBAPS_WAIT_LIMIT_NS=1000000ull", "-DBAPS_TEST_SKIP_LOAD=1"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xptxas", "-v",
    # inline variables (the count of launches, the lock of the set-up) belong to one library, also where a process loads two builds
    "-Xcompiler", "-fno-gnu-unique",
]
UNITS = ["baps_lib.cu", "baps_serving.cu"]
MARSHAL = os.path.join(_HERE, "_serving.so")


def _sources(path: str, seen=None):
    """``path`` and every file that it includes by a quoted name, however deep."""
    seen = set() if seen is None else seen
    path = os.path.normpath(path)
    if path not in seen:
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^\s*#include "([^"]+)"', f.read(), re.M):
                _sources(os.path.join(os.path.dirname(path), name), seen)
    return seen


def _portable(cmd) -> str:
    """A command as one line that is the same wherever the tree stands."""
    return " ".join(cmd).replace(os.path.normpath(os.path.join(_HERE, "..")) + os.sep, "")


def _is_current(path: str, log: str, line: str, sources) -> bool:
    """Whether ``path`` is there, no older than its sources, and made by this command (the first line of its log)."""
    if not (os.path.exists(path) and os.path.exists(log)) or os.path.getmtime(path) < max(os.path.getmtime(p) for p in sources):
        return False
    with open(log) as f:
        return f.readline() == line + "\n"


def _compile_unit(unit: str, lib: str, extra_flags, force: bool):
    """One object file next to the library, if it is missing, older than a source or made by another command; returns
    (path, compiler's output)."""
    obj = f"{lib}.{os.path.splitext(unit)[0]}.o"
    src = os.path.join(CSRC, unit)
    log = obj + ".log"
    cmd = [os.environ.get("NVCC", "nvcc"), *NVCC_FLAGS, *extra_flags, "-c", "-o", obj + ".tmp", src]
    if not force and _is_current(obj, log, _portable(cmd), _sources(src)):
        with open(log) as f:
            return obj, f.read()
    res = subprocess.run(cmd, capture_output=True, text=True)
    text = _portable(cmd) + "\n" + res.stdout + res.stderr
    if res.returncode != 0:
        sys.stderr.write(text)
        raise RuntimeError(f"nvcc failed on {unit}")
    with open(log, "w") as f:
        f.write(text)
    os.replace(obj + ".tmp", obj)
    return obj, text


def _compile(lib: str, extra_flags, log_name: str, force: bool, verbose: bool) -> str:
    key = _portable([os.environ.get("NVCC", "nvcc"), *NVCC_FLAGS, *extra_flags, *UNITS])
    path = os.path.join(_HERE, log_name)
    if not force and _is_current(lib, path, key, {p for u in UNITS for p in _sources(os.path.join(CSRC, u))}):
        return lib
    with ThreadPoolExecutor(len(UNITS)) as pool:
        done = list(pool.map(lambda u: _compile_unit(u, lib, extra_flags, force), UNITS))
    cmd = [os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "--shared", "-o", lib, *(o for o, _ in done)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    log = "".join(t for _, t in done) + _portable(cmd) + "\n" + res.stdout + res.stderr
    with open(path, "w") as f:
        f.write((key if res.returncode == 0 else "failed") + "\n" + log)
    if verbose or res.returncode != 0:
        sys.stderr.write(log)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed linking {os.path.basename(lib)} (see {log_name})")
    return lib


def _compile_marshal(force: bool) -> None:
    src = os.path.join(CSRC, "serving_marshal.cpp")
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"))
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-Wall", "-Wextra", "-shared", "-fPIC",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + sysconfig.get_path("include"),
           "-isystem", root + "/include", "-isystem", root + "/include/torch/csrc/api/include", "-isystem", cuda + "/include",
           "-o", MARSHAL + ".tmp", src, "-L" + root + "/lib", "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    # (compiled against the C++ interfaces of this torch and this Python)
    key, log = f"torch {torch.__version__}, Python {sys.version.split()[0]}: " + _portable(cmd), MARSHAL + ".o.log"
    if not force and _is_current(MARSHAL, log, key, _sources(src)):
        return
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(" ".join(cmd) + "\n" + res.stdout + res.stderr)
        raise RuntimeError("the C++ compiler failed on serving_marshal.cpp")
    with open(log, "w") as f:
        f.write(key + "\n" + res.stdout + res.stderr)
    os.replace(MARSHAL + ".tmp", MARSHAL)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library and the binding's module if they are missing, older than any source or made by another command (other
    flags, another compiler, torch or Python); return the library's path."""
    _compile_marshal(force)
    extra = os.environ.get("BAPS_NVCC_EXTRA", "").split()       # developer switch, e.g. -DNAME=1
    return _compile(LIB, extra, "build.log", force, verbose)


def build_wait_test(force: bool = False, verbose: bool = False) -> str:
    """Compile the wait-test build of the library (see WAIT_TEST_LIB)."""
    return _compile(WAIT_TEST_LIB, WAIT_TEST_FLAGS, "build_waittest.log", force, verbose)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
    print(build_wait_test(force="--force" in sys.argv, verbose=False))
