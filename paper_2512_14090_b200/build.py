"""Builds libaiq.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
import contextlib
import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
ROOT = os.path.dirname(PKG_DIR)
BUILD_DIR = os.path.join(ROOT, "_build")
LIB_PATH = os.path.join(PKG_DIR, "libaiq.so")
CALL_SRC = os.path.join(CSRC, "mxcall.c")
CALL_PATH = os.path.join(PKG_DIR, "_mxcall" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc():
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the library cannot be built")
    return exe


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build_call(force=False):
    """The CPython entry to the microscaled calls, against libaiq.so beside it.  Where it cannot be built (no C compiler, no Python header, or one
    that fails) the binding goes through ctypes; a module built from other sources goes, since its calls may not be the library's."""
    if not force and not _stale(CALL_PATH, [CALL_SRC, os.path.join(ROOT, "include", "aiq.h")]):
        return CALL_PATH
    with contextlib.suppress(FileNotFoundError):
        os.remove(CALL_PATH)
    include = sysconfig.get_paths()["include"]
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None or not os.path.exists(os.path.join(include, "Python.h")):
        return None
    cmd = [cc, "-O2", "-shared", "-fPIC", "-I", include, CALL_SRC, "-o", CALL_PATH, "-L", PKG_DIR, "-l:libaiq.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        warnings.warn(f"compiling {CALL_SRC} failed; the microscaled calls go through ctypes:\n{r.stdout}\n{r.stderr}")
        return None
    return CALL_PATH


def build(force=False, verbose=False):
    """Compile every .cu under csrc/, link libaiq.so and compile its CPython entry.  Returns the library path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers.append(os.path.join(ROOT, "include", "aiq.h"))
    if not force and not _stale(LIB_PATH, sources() + headers):
        build_call()
        return LIB_PATH
    nvcc = _nvcc()
    objs, todo = [], []
    for src in sources():
        obj = os.path.join(BUILD_DIR, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or _stale(obj, [src] + headers):
            todo.append((src, obj))

    def compile_one(job):
        src, obj = job
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        return r.stderr

    with ThreadPoolExecutor(max_workers=max(1, min(8, len(todo)))) as ex:
        logs = list(ex.map(compile_one, todo))
    if verbose:
        for log in logs:
            sys.stderr.write(log)
    if todo or force or _stale(LIB_PATH, objs):
        cmd = [nvcc, "-shared", "-o", LIB_PATH] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    build_call(force)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
