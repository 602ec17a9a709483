"""Builds the CUDA extension (a plain C-ABI shared library) in-tree for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB_DIR = os.path.join(_HERE, "_lib")
LIB_PATH = os.path.join(LIB_DIR, "libobf_b200.so")
SOURCES = ["obf_api.cu", "obf_attend.cu", "obf_quant.cu"]


def _newest_source_mtime() -> float:
    t = os.path.getmtime(os.path.join(ROOT, "include", "obf.h"))
    for f in os.listdir(CSRC):
        if f.endswith((".cu", ".cuh", ".h")):
            t = max(t, os.path.getmtime(os.path.join(CSRC, f)))
    return t


def _nvcc():
    return [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a"]


def compile_command(source: str, out: str, verbose: bool = False):
    """Compiles one source file to an object file."""
    cmd = _nvcc() + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC,-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                     "-c", "-o", out]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    return cmd + [os.path.join(CSRC, source)]


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(LIB_DIR, exist_ok=True)
    if not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _newest_source_mtime():
        return LIB_PATH
    tmp = LIB_PATH + ".tmp%d" % os.getpid()
    objects = ["%s.%d.o" % (tmp, i) for i in range(len(SOURCES))]
    try:
        jobs = [subprocess.Popen(compile_command(s, o, verbose), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                for s, o in zip(SOURCES, objects)]
        said = [j.communicate()[0] for j in jobs]
        ok = all(j.returncode == 0 for j in jobs)
        if ok:
            r = subprocess.run(_nvcc() + ["--shared", "-o", tmp] + objects, capture_output=True, text=True)
            said.append(r.stdout + r.stderr)
            ok = r.returncode == 0
        if verbose or not ok:
            sys.stderr.write("".join(said))
        if not ok:
            raise RuntimeError("nvcc failed building %s" % LIB_PATH)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
