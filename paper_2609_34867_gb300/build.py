"""Builds libp4q.so (the sm_103a kernels behind include/p4q.h) in-tree with nvcc.

Each .cu under csrc/ is compiled in parallel for sm_103a only, then linked
into paper_2609_34867_gb300/lib/libp4q.so; the Python module of csrc/p4q_call.c, which
marshals the calls of a decode step, goes beside it where there are Python's headers to compile
it (without it the binding marshals these calls through ctypes). No fast-math: the quantizer and the
cosine rely on IEEE-rounded fp32 division and square root.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBDIR = os.path.join(PKG, "lib")
LIB = os.path.join(LIBDIR, "libp4q.so")
CALL = os.path.join(LIBDIR, "p4q_call.so")
GENCODE = "-gencode=arch=compute_103a,code=sm_103a"


def nvcc() -> str:
    home = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    path = os.path.join(home, "bin", "nvcc")
    return path if os.path.exists(path) else (shutil.which("nvcc") or "nvcc")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + \
        glob.glob(os.path.join(INCLUDE, "*.h")) + glob.glob(os.path.join(CSRC, "*.c"))


def python_headers():
    """The folder of Python.h, None where Python has none (they are a package of their own in most systems)."""
    path = sysconfig.get_paths()["include"]
    return path if os.path.exists(os.path.join(path, "Python.h")) else None


def up_to_date() -> bool:
    built = [LIB, CALL] if python_headers() else [LIB]
    if not all(os.path.exists(p) for p in built):
        return False
    t = min(os.path.getmtime(p) for p in built)
    return all(os.path.getmtime(p) <= t for p in _deps())


def _start_call(verbose: bool):
    """The compiler at work on csrc/p4q_call.c and the file that it writes; None without Python's headers."""
    headers = python_headers()
    if headers is None:
        print(f"no Python.h in {sysconfig.get_paths()['include']}: calls of a decode step go through ctypes", file=sys.stderr)
        return None
    tmp = f"{CALL}.tmp{os.getpid()}"
    cmd = [shutil.which("gcc") or "cc", "-O2", "-Wall", "-shared", "-fPIC", "-I", headers, "-I", INCLUDE,
           os.path.join(CSRC, "p4q_call.c"), "-o", tmp]
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True), tmp


def _finish_call(started) -> None:
    if started is None:
        if os.path.exists(CALL):  # (of another source, perhaps)
            os.remove(CALL)
        return
    p, tmp = started
    out, _ = p.communicate()
    if p.returncode:
        raise RuntimeError(f"the C compiler failed for p4q_call.c (libp4q.so is built):\n{out}")
    os.replace(tmp, CALL)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    objdir = os.path.join(LIBDIR, "obj")
    os.makedirs(objdir, exist_ok=True)
    flags = [GENCODE, "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC,
             "--expt-relaxed-constexpr"]
    if ptxas_info:
        flags += ["-Xptxas", "-v"]
    procs = []
    objs = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc()] + flags + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    call = _start_call(verbose)
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if out and (verbose or ptxas_info or p.returncode):
            print(out, file=sys.stderr)
        if p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"nvcc failed for {failed}")
    tmp = LIB + f".tmp{os.getpid()}"
    # every symbol resolved at link time (a missing definition fails here, not at load)
    subprocess.run([nvcc(), GENCODE, "-shared", "-Xlinker", "--no-undefined", "-o", tmp] + objs, check=True)
    os.replace(tmp, LIB)
    _finish_call(call)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv, ptxas_info="--ptxas" in sys.argv)
    print(LIB)
