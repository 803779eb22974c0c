"""Build the CUDA library in-tree: ``python -m paper_2609_04098_b200.build``.

nvcc cross-compiles for sm_100a without a GPU.  The shared object lands next to
this file so that it travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libnvfp4_b200.so")
API_H = os.path.join("..", "..", "include", "nvfp4.h")
SOURCES = {        # translation unit -> the headers it includes
    "nvfp4_api.cu": ["gemm.cuh", "decode.cuh", "quantize.cuh", "recurrence.cuh", "ptx.cuh", "host.h", API_H],
    "gdn_api.cu": ["gdn.cuh", "gdn_chunk.cuh", "ptx.cuh", "host.h", API_H],
}


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _object(source: str) -> str:
    return os.path.join(CSRC, os.path.splitext(source)[0] + ".o")


def _stale(target: str, sources) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in list(sources) + [os.path.abspath(__file__)])


def _run(cmd, verbose: bool) -> None:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed (%d)" % res.returncode)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile what is out of date (one nvcc process per translation unit, side by side) and link the library."""
    all_files = {os.path.join(CSRC, f) for s, deps in SOURCES.items() for f in [s] + deps}
    if not force and not _stale(LIB, all_files):
        return LIB
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    pid = os.getpid()

    def compile_one(source: str) -> None:
        obj = _object(source)
        if force or _stale(obj, [os.path.join(CSRC, f) for f in [source] + SOURCES[source]]):
            tmp = obj[:-2] + ".tmp%d.o" % pid
            _run([nvcc_path()] + flags + ["-c", "-o", tmp, os.path.join(CSRC, source)], verbose)
            os.replace(tmp, obj)

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        list(pool.map(compile_one, SOURCES))
    tmp = LIB + ".tmp%d" % pid
    _run([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "-o", tmp]
         + [_object(s) for s in SOURCES], False)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
