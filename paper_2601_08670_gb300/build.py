"""In-tree build of libpced.so (the sm_103a decoding library) with nvcc.

Translation units compile in parallel, then link into one shared library
under ``paper_2601_08670_gb300/_lib``.  The library links the CUDA runtime
statically and fetches the driver's tensor-map encoder at run time, so it has
no link-time dependency on libcuda and none on PyTorch.  Beside it g++ compiles
the binding's CPython module (calls.cpp) against the installed PyTorch; where
that fails, the library is there all the same.
"""
from __future__ import annotations

import importlib.metadata
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
           "step.cu", "partition.cu", "host.cu", "kv_append.cu", "block_select.cu", "paged_attention.cu", "logits.cu",
           "kv_append8.cu", "paged_attention8.cu", "sample.cu", "sample_bf16.cu"]
CALLS = "pced_calls.so"


def _calls_for() -> str:
    """What the binding's module is compiled against: of another PyTorch or Python it has to be built anew."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch = "none"
    return f"torch {torch} {sysconfig.get_config_var('SOABI')}"


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


def _newest(files) -> float:
    return max(os.path.getmtime(f) for f in [*files, os.path.join(ROOT, "include", "pced.h")])


def _fresh(built: str, newest: float) -> bool:
    return os.path.exists(built) and os.path.getmtime(built) >= newest


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False, checked: bool = False) -> str:
    """Compiles libpced.so if a source is newer, and the binding's module if its source is, or if PyTorch or Python
    is another; `checked` builds the bounds-checked library (-DPCED_BOUNDS_CHECK) into its own folder.  A module that
    cannot be built is reported when the library is linked."""
    libdir, lib = (CHECKED_LIBDIR, CHECKED_LIB) if checked else (LIBDIR, LIB)
    os.makedirs(libdir, exist_ok=True)
    calls, stamp = os.path.join(libdir, CALLS), os.path.join(libdir, "pced_calls.txt")
    source = os.path.join(CSRC, "calls.cpp")
    others = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "calls.cpp"]
    need_lib = force or not _fresh(lib, _newest(others))
    need_calls = force or not _fresh(calls, _newest([source])) or not os.path.exists(stamp)
    if not need_calls:
        with open(stamp) as f:
            need_calls = f.read() != _calls_for()
    if not need_lib and not need_calls:
        return lib
    procs = []
    objs = []
    for src in SOURCES if need_lib else []:
        obj = os.path.join(libdir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = ["nvcc", *ARCH, *FLAGS, *(["-DPCED_BOUNDS_CHECK"] if checked else []), "-c", os.path.join(CSRC, src),
               "-o", obj]
        if ptxas_info:
            cmd += ["-Xptxas", "-v"]
        procs.append((src, _start(cmd)))
    calls_failed = None
    if need_calls:
        try:
            calls_compile, calls_link = _calls_commands(libdir)
            procs.append(("calls.cpp", _start(calls_compile)))
        except (ImportError, OSError) as e:  # no PyTorch, no compiler
            calls_failed = e
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(f"--- {src}\n{out}")
        if p.returncode != 0:
            failed.append(src)
    if "calls.cpp" in failed:
        failed.remove("calls.cpp")
        calls_failed = RuntimeError("g++ failed")
    if failed:
        raise RuntimeError(f"compilation failed for {failed}")
    if need_lib:
        tmp = lib + f".tmp{os.getpid()}"
        subprocess.check_call(["nvcc", *ARCH, "-shared", "-Xlinker", "-soname=libpced.so", "-o", tmp, *objs, "-cudart",
                               "static"])
        os.replace(tmp, lib)
    if need_calls and calls_failed is None:
        try:
            subprocess.check_call(calls_link)
            os.replace(calls_link[calls_link.index("-o") + 1], calls)
            with open(stamp, "w") as f:
                f.write(_calls_for())
        except (subprocess.CalledProcessError, OSError) as e:
            calls_failed = e
    if calls_failed is not None:
        if os.path.exists(calls):
            os.remove(calls)  # (one that is out of date: of another header or another PyTorch)
        raise RuntimeError(f"{lib} is built, the binding's module (calls.cpp) is not: {calls_failed}") from calls_failed
    return lib


if __name__ == "__main__":
    build(force=True, verbose=True, ptxas_info="-v" in sys.argv)
