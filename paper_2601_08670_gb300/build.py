"""In-tree build of libpced.so (the sm_103a decoding library) with nvcc.

Translation units compile in parallel, then link into one shared library
under ``paper_2601_08670_gb300/_lib``.  The library links the CUDA runtime
statically and fetches the driver's tensor-map encoder at run time, so it has
no link-time dependency on libcuda.  Beside it g++ compiles the binding's
CPython module (calls.cpp) against the installed PyTorch.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "_lib")
LIB = os.path.join(LIBDIR, "libpced.so")
# the bounds-checked build: every guarded index outside its buffer sets
# PCED_DEV_BOUNDS in the status word and skips the access
CHECKED_LIBDIR = os.path.join(HERE, "_lib_checked")
CHECKED_LIB = os.path.join(CHECKED_LIBDIR, "libpced.so")
ROOT = os.path.dirname(HERE)
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-I", os.path.join(ROOT, "include")]
SOURCES = ["attention.cu", "attention_noalloc.cu", "lm_head.cu", "lm_head_pair.cu", "select.cu", "adacad.cu", "aggregate.cu", "relevance.cu",
           "step.cu", "partition.cu", "host.cu", "kv_append.cu", "block_select.cu", "paged_attention.cu", "logits.cu"]


CALLS = "pced_calls.so"


def _calls_commands(libdir: str) -> tuple:
    """g++ commands that compile the binding's CPython module and link it to the library beside it."""
    import torch
    home = os.path.dirname(torch.__file__)
    include = [os.path.join(ROOT, "include"), os.path.join(home, "include"), sysconfig.get_paths()["include"],
               os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    obj = os.path.join(libdir, "calls.o")
    compile_ = ["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                *[f for p in include for f in ("-I", p)], "-c", os.path.join(CSRC, "calls.cpp"), "-o", obj]
    link = ["g++", "-shared", "-o", os.path.join(libdir, CALLS + f".tmp{os.getpid()}"), obj, "-L", libdir, "-lpced",
            "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN"]
    return compile_, link


def _deps():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "pced.h")]
    return max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False, checked: bool = False) -> str:
    """Compiles libpced.so if a source is newer; `checked` builds the
    bounds-checked library (-DPCED_BOUNDS_CHECK) into its own folder."""
    libdir, lib = (CHECKED_LIBDIR, CHECKED_LIB) if checked else (LIBDIR, LIB)
    os.makedirs(libdir, exist_ok=True)
    calls = os.path.join(libdir, CALLS)
    if not force and all(os.path.exists(f) and os.path.getmtime(f) >= _deps() for f in (lib, calls)):
        return lib
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(libdir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = ["nvcc", *ARCH, *FLAGS, *(["-DPCED_BOUNDS_CHECK"] if checked else []), "-c", os.path.join(CSRC, src),
               "-o", obj]
        if ptxas_info:
            cmd += ["-Xptxas", "-v"]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    calls_compile, calls_link = _calls_commands(libdir)
    procs.append(("calls.cpp", subprocess.Popen(calls_compile, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(f"--- {src}\n{out}")
        if p.returncode != 0:
            failed.append(src)
    if failed:
        raise RuntimeError(f"compilation failed for {failed}")
    tmp = lib + f".tmp{os.getpid()}"
    subprocess.check_call(["nvcc", *ARCH, "-shared", "-Xlinker", "-soname=libpced.so", "-o", tmp, *objs, "-cudart",
                           "static"])
    os.replace(tmp, lib)
    subprocess.check_call(calls_link)
    os.replace(calls_link[calls_link.index("-o") + 1], calls)
    return lib


if __name__ == "__main__":
    build(force=True, verbose=True, ptxas_info="-v" in sys.argv)
