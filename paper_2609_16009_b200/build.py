"""Builds the C-ABI library ``libnm.so`` in-tree with nvcc for sm_100a.

Run as ``python paper_2609_16009_b200/build.py`` (as a script: importing the package needs the library this builds).  Object files go to ``build/`` at the
repository root; the shared library is written next to this file.  Only changed sources are
recompiled (mtime against every header).  ``--check`` builds the debug library ``libnm_check.so`` instead (the same
sources with ``-DNM_BOUNDS_CHECK``).
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "build", "nm")
LIB = os.path.join(PKG, "libnm.so")
CALLS_SRC = os.path.join(CSRC, "nm_python.c")
CALLS = os.path.join(PKG, "_nm_calls" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--threads", "2"]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("nvcc not found")


def build_calls() -> str | None:
    """The extension module through which the binding makes its short calls (csrc/nm_python.c); None where Python's headers are missing: they go through ctypes then."""
    include = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(include, "Python.h")):
        return None
    if not os.path.exists(CALLS) or os.path.getmtime(CALLS) < os.path.getmtime(CALLS_SRC):
        tmp = CALLS + f".tmp{os.getpid()}"
        r = subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", include, CALLS_SRC, "-o", tmp], capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("gcc failed on nm_python.c")
        os.replace(tmp, CALLS)
    return CALLS


def build(verbose: bool = False, force: bool = False, ptxas_info: bool = False, check: bool = False) -> str:
    """check=True: the debug build (libnm_check.so, -DNM_BOUNDS_CHECK: the narrow-product kernels check their hand-indexed
    global accesses against the operands' extents); its objects live in their own directory."""
    OBJ = os.path.join(ROOT, "build", "nm_check" if check else "nm")
    LIB = os.path.join(PKG, "libnm_check.so" if check else "libnm.so")
    os.makedirs(OBJ, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)
    nvcc = _nvcc()
    jobs = []
    objs = []
    for src in sources:
        obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        stale = force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), newest_header)
        if stale:
            cmd = [nvcc, *NVCC_FLAGS, *(["-DNM_BOUNDS_CHECK"] if check else []), "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
            if ptxas_info:
                cmd[1:1] = ["-Xptxas", "-v"]
            jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose or r.returncode != 0 or ptxas_info:
                sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {cmd[-3]}")
    if jobs or not os.path.exists(LIB):
        tmp = LIB + f".tmp{os.getpid()}"
        cmd = [nvcc, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
        os.replace(tmp, LIB)
    if not check:
        build_calls()
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv, ptxas_info="--ptxas" in sys.argv, check="--check" in sys.argv))
