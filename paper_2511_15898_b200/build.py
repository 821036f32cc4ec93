"""Compile the CUDA library (sm_100a) into paper_2511_15898_b200/libgr_b200.so."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgr_b200.so")
LIB_CHECK = os.path.join(HERE, "libgr_b200_check.so")      # the bounds-checked build (-DGR_CHECK)
OBJ = os.path.join(HERE, "_build")
SOURCES = ["gr_api.cu", "gr_alpha.cu", "gr_static.cu", "gr_scan.cu", "gr_solve.cu", "gr_fast.cu", "gr_fast_n4.cu", "gr_fast_n8.cu",
           "gr_fast_n16.cu", "gr_fast_n8w.cu", "gr_fast_n16w.cu", "gr_fast_c24.cu", "gr_fullsort.cu", "gr_verify.cu", "gr_beam.cu",
           "gr_states.cu", "gr_blocks.cu", "gr_cache.cu", "gr_attend.cu", "gr_logprobs.cu"]
HEADERS = [os.path.join(CSRC, "gr_common.cuh"), os.path.join(CSRC, "gr_prep.cuh"), os.path.join(CSRC, "gr_quad.cuh"), os.path.join(CSRC, "gr_scan.cuh"), os.path.join(CSRC, "gr_fast.cuh"), os.path.join(CSRC, "gr_verify.cuh"), os.path.join(CSRC, "gr_list.cuh"), os.path.join(CSRC, "gr_cache.cuh"), os.path.join(CSRC, "gr_host.h"),
           os.path.join(ROOT, "include", "gr.h")]


# The binding's short way for tensors: a Python module on torch's headers, which the package does without where it cannot be compiled.
# Beside it stands what it was compiled from (its sources and torch), in words.
TENSORS_SOURCE = os.path.join(CSRC, "gr_tensors.cpp")
TENSORS = os.path.join(HERE, "_tensors.so")


def _tensors_of() -> str:
    """What a module compiled now would be compiled from."""
    import hashlib
    try:
        from torch import __version__ as torch_version
    except ImportError:
        torch_version = None
    h = hashlib.sha256()
    for path in (TENSORS_SOURCE, os.path.join(ROOT, "include", "gr.h")):
        with open(path, "rb") as f:
            h.update(f.read())
    return f"torch {torch_version} python {sys.version.split()[0]} sources {h.hexdigest()}"


def _tensors_fresh() -> bool:
    """Whether the module, or the note that it could not be compiled, is of the present sources."""
    try:
        with open(TENSORS + ".txt") as f:
            of, state = f.read().split("\n")[:2]
    except (OSError, ValueError):
        return False
    return of == _tensors_of() and (state == "failed" or os.path.exists(TENSORS))


def _start_tensors():
    """The started compilation of the module, or what kept it from starting."""
    import sysconfig
    try:
        import torch
        from torch.utils.cpp_extension import include_paths
    except ImportError as e:
        return str(e)
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            f'-DGR_TORCH_VERSION="{torch.__version__}"']
           + [a for p in include_paths() + [sysconfig.get_paths()["include"], os.path.join(_cuda_home(), "include")] for a in ("-isystem", p)]
           + ["-I", os.path.join(ROOT, "include"), TENSORS_SOURCE, "-L" + lib, "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath," + lib, "-o", TENSORS])
    try:
        return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    except OSError as e:
        return str(e)


def _finish_tensors(started):
    if isinstance(started, str):
        out = started
    else:
        out, _ = started.communicate()
    done = not isinstance(started, str) and started.returncode == 0
    if not done:
        sys.stderr.write(f"{os.path.basename(TENSORS_SOURCE)} could not be compiled, the binding's calls go the way in Python:\n{out}\n")
        if os.path.exists(TENSORS):
            os.remove(TENSORS)
    with open(TENSORS + ".txt", "w") as f:
        f.write(_tensors_of() + ("\nbuilt\n" if done else "\nfailed\n"))


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _cuda_home() -> str:
    return os.path.dirname(os.path.dirname(_nvcc())) if os.path.sep in _nvcc() else "/usr/local/cuda"


def needs_build(check: bool = False) -> bool:
    lib = LIB_CHECK if check else LIB
    if not os.path.exists(lib):
        return True
    if not check and not _tensors_fresh():
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False, check: bool = False) -> str:
    """Compile each source to an object (in parallel; objects newer than every source and header are kept),
    then link the shared library.  check=True builds the bounds-checked variant (-DGR_CHECK: every access through a
    pointer into shared memory, the workspace records or the params block is range-checked, an out-of-range access
    is skipped and reported as status GR_CHECK_FAILED) into a library file of its own; it is for tests only."""
    LIB = LIB_CHECK if check else globals()["LIB"]
    OBJ = globals()["OBJ"] + ("_check" if check else "")
    if not force and not needs_build(check):
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if check:
        flags += ["-DGR_CHECK"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    hdr_time = max(os.path.getmtime(h) for h in HEADERS)
    jobs = []
    objs = []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(OBJ, s[:-3] + ".o")
        objs.append(obj)
        fresh = (not force and not verbose and os.path.exists(obj)
                 and os.path.getmtime(obj) > max(os.path.getmtime(src), hdr_time))
        if not fresh:
            jobs.append((s, subprocess.Popen([_nvcc()] + flags + ["-c", src, "-o", obj], stdout=subprocess.PIPE,
                                             stderr=subprocess.STDOUT, text=True)))
    tensors = _start_tensors() if not check and (force or not _tensors_fresh()) else None
    failed = []
    for s, proc in jobs:
        out, _ = proc.communicate()
        if verbose:
            sys.stderr.write(out)
        if proc.returncode != 0:
            failed.append(s + ":\n" + out)
    if tensors is not None:
        _finish_tensors(tensors)
    if failed:
        raise RuntimeError("nvcc failed:\n" + "\n".join(failed))
    res = subprocess.run([_nvcc(), "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a"]
                         + objs + ["-ldl", "-o", LIB], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
