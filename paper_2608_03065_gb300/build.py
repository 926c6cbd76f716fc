"""Builds libpsc_gb300.so in-tree: host C++ (g++) + CUDA for sm_103a (nvcc), linked
with nvcc (static CUDA runtime).  Translation units compile in parallel."""
from __future__ import annotations

import concurrent.futures as cf
import fcntl
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpsc_gb300.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

CXX_SOURCES = ["grammar.cpp", "lexer.cpp", "lalr.cpp", "classifier.cpp", "bottomup.cpp", "persist.cpp"]
CU_SOURCES = ["psc_capi.cu", "process.cu", "sample.cu", "head.cu", "norm.cu", "mx4.cu",
              "mx4_head.cu"]
GENCODE = "arch=compute_103a,code=sm_103a"
# the binding's Python module, by the interpreter that it is built for (psc.py does without it where Python.h is missing)
MARSHAL = os.path.join(HERE, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build the library")


def _stale(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles what is stale and links the library.  Processes that build at
    the same time (one per rank) take turns on a lock file."""
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        return _build_locked(force, verbose)


def _build_locked(force: bool, verbose: bool) -> str:
    headers = [os.path.join(CSRC, "psc_internal.h"), os.path.join(INCLUDE, "psc.h")]
    ops_headers = [os.path.join(CSRC, f) for f in ("ops_common.cuh", "mx4.cuh", "tcgen05.cuh")]
    ops_headers += [os.path.join(INCLUDE, f) for f in ("psc_ops.h", "psc_mx4.h", "psc_norm.h")]
    nvcc = _nvcc()
    jobs = []
    objs = []
    for src in CXX_SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src + ".o")
        objs.append(o)
        if force or _stale(o, [s] + headers):
            jobs.append(["g++", "-O2", "-std=c++17", "-fPIC", "-pthread", "-Wall", "-Wno-sign-compare",
                         "-I", INCLUDE, "-c", s, "-o", o])
    for src in CU_SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src + ".o")
        objs.append(o)
        if force or _stale(o, [s] + headers + ops_headers):
            jobs.append([nvcc, "-gencode", GENCODE, "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
                         "-I", INCLUDE, "-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"build failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr)
        return r

    def put(target, cmd):
        """Makes a file that processes may have loaded, or may load meanwhile: beside it, then in its place."""
        tmp = target + f".{os.getpid()}.tmp"
        run(cmd + ["-o", tmp])
        os.replace(tmp, target)

    python = sysconfig.get_paths()["include"]
    marshal = os.path.join(CSRC, "marshal.cpp")
    with cf.ThreadPoolExecutor(max_workers=len(jobs) + 1) as ex:
        waits = [ex.submit(run, cmd) for cmd in jobs]
        if os.path.exists(os.path.join(python, "Python.h")) and (force or _stale(MARSHAL, [marshal])):
            waits.append(ex.submit(put, MARSHAL, ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", python, marshal]))
        for w in waits:
            w.result()
    if force or jobs or _stale(LIB, objs):
        put(LIB, [nvcc, "-shared", "-gencode", GENCODE] + objs + ["-lpthread", "-ldl"])
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
