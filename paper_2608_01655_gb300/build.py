"""In-tree build of libprefixplace.so for sm_103a (nvcc, no CMake).

Each .cu file under csrc/ is compiled in parallel, then linked into one
shared library next to this file; the benchmark's bandwidth probe
(probe/pp_probe.cu) becomes a library of its own, libpp_probe.so.  csrc/pp_call.c
is a Python extension with the cache's calls, _pp_call, where Python's headers
are installed and a C compiler takes it; the binding does without.  The CUDA
runtime is linked statically, so the libraries need only the driver at run
time and no torch symbols.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libprefixplace.so")
PROBE_SRC = os.path.join(HERE, "probe", "pp_probe.cu")
PROBE_LIB = os.path.join(HERE, "libpp_probe.so")   # the benchmark's bandwidth probe, not the planner
CALL_SRC = os.path.join(CSRC, "pp_call.c")
CALL_LIB = os.path.join(HERE, "_pp_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC]


def _nvcc():
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libprefixplace")
    return exe


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    files = sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    files.append(os.path.join(INCLUDE, "prefixplace.h"))
    return files


def _python_include():
    """Where Python.h is, None if it is not installed."""
    path = sysconfig.get_paths()["include"]
    return path if os.path.exists(os.path.join(path, "Python.h")) else None


def up_to_date() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(PROBE_LIB):
        return False
    t = os.path.getmtime(LIB)
    tp = os.path.getmtime(PROBE_LIB)
    return all(os.path.getmtime(f) <= t for f in _deps()) and \
        all(os.path.getmtime(f) <= tp for f in (PROBE_SRC, os.path.join(INCLUDE, "pp_probe.h")))


def _build_call(force: bool = False):
    """The extension module, if it is missing or older than its sources.  It is optional: without Python's headers
    there is none, and where it does not compile the build goes on, with a warning and none that is out of date."""
    include = _python_include()
    if not include:
        return
    if not force and os.path.exists(CALL_LIB) and all(
            os.path.getmtime(f) <= os.path.getmtime(CALL_LIB) for f in (CALL_SRC, os.path.join(INCLUDE, "prefixplace.h"))):
        return
    tmp = CALL_LIB + f".tmp{os.getpid()}"
    cmd = [shutil.which("gcc") or "cc", "-O2", "-Wall", "-shared", "-fPIC", "-I" + include, "-I" + INCLUDE, CALL_SRC, "-o", tmp]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
        why = r.stdout + r.stderr if r.returncode != 0 else None
    except OSError as e:
        why = str(e)
    if why is None:
        os.replace(tmp, CALL_LIB)
        return
    for path in (tmp, CALL_LIB):
        if os.path.exists(path):
            os.remove(path)
    warnings.warn(f"{os.path.basename(CALL_SRC)} does not compile: the cache's calls go by ctypes\n{why}")


def build(force: bool = False, verbose: bool = False, extra=()) -> str:
    if not force and up_to_date():
        _build_call()
        return LIB
    nvcc = _nvcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *ARCH, *FLAGS, *extra, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr)
        return obj

    def build_probe():
        tmp = PROBE_LIB + f".tmp{os.getpid()}"
        cmd = [nvcc, *ARCH, *FLAGS, *extra, "-shared", PROBE_SRC, "-o", tmp]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {PROBE_SRC}:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, PROBE_LIB)

    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        probe, call = ex.submit(build_probe), ex.submit(_build_call, force)
        objs = list(ex.map(compile_one, sources()))
        probe.result()
        call.result()
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
