"""Build libmc.so (the C-ABI library) in-tree with nvcc for sm_103a.

Every translation unit is compiled in parallel to an object file under
``paper_2410_06270_gb300/_build/`` and linked into ``_build/libmc.so``.  Objects
are rebuilt when their source or any header is newer.  No cmake, no torch
extension machinery: the library has a plain C ABI.  Beside it, the marshalling of
the calls that a decode step makes is a small CPython extension.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libmc.so")
BIND = os.path.join(BUILD, "_mcbind.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc():
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else (shutil.which("nvcc") or "nvcc")


def _headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(INCLUDE, "*.h"))


def _stale(obj, src, hdr_mtime):
    if not os.path.exists(obj):
        return True
    t = os.path.getmtime(obj)
    return t < os.path.getmtime(src) or t < hdr_mtime


def build(verbose: bool = False, force: bool = False, ptxas_verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))
    hdr_mtime = max([os.path.getmtime(h) for h in _headers()] + [0])
    common = ["-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
    jobs = []
    objs = []
    for src in srcs:
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        objs.append(obj)
        if force or _stale(obj, src, hdr_mtime):
            cmd = [nvcc] + common + ARCH + ["-lineinfo", "-c", src, "-o", obj]
            if src.endswith(".cu"):
                cmd += ["--expt-relaxed-constexpr"]
                if ptxas_verbose:
                    cmd += ["-Xptxas", "-v"]
            else:
                cmd = [nvcc] + common + ["-x", "c++", "-c", src, "-o", obj]
            jobs.append(cmd)
    if jobs:
        with cf.ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 4)) as ex:
            results = list(ex.map(lambda c: subprocess.run(c, capture_output=True, text=True), jobs))
        for cmd, r in zip(jobs, results):
            if verbose or ptxas_verbose or r.returncode:
                sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
            if r.returncode:
                raise RuntimeError("nvcc failed for " + cmd[-3 if cmd[-1].endswith('.o') else -1])
    if jobs or not os.path.exists(LIB):
        tmp = LIB + ".tmp%d" % os.getpid()
        subprocess.check_call([nvcc, "-shared"] + ARCH + ["-o", tmp] + objs + ["-lcudart"])
        os.replace(tmp, LIB)
    _build_binding()
    return LIB


def _build_binding() -> None:
    """The CPython extension that marshals the calls of a decode step (host code, gcc)."""
    src = os.path.join(HERE, "bind", "mc_bind.c")
    if os.path.exists(BIND) and os.path.getmtime(BIND) >= max(os.path.getmtime(src), *[os.path.getmtime(h) for h in _headers()]):
        return
    tmp = BIND + ".tmp%d" % os.getpid()
    subprocess.check_call(["gcc", "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-I", INCLUDE, src,
                           "-o", tmp])
    os.replace(tmp, BIND)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv, ptxas_verbose="--ptxas" in sys.argv))
