"""Builds the C-ABI shared library in-tree with nvcc for sm_100a.

    python -m paper_2505_19578_b200.build [--force] [--verbose] [--debug]

Output: paper_2505_19578_b200/libshareprefill.so (cudart linked statically; the
driver API is resolved at run time, so the library loads on a machine without a
GPU driver), and paper_2505_19578_b200/_decode_calls.so, the Python entry of the
decode-side calls (g++ against torch's headers; without torch it is left out).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libshareprefill.so")
LIB_DEBUG = os.path.join(HERE, "libshareprefill_debug.so")   # the same sources with -DSP_DEBUG: range-checked indices
SOURCES = ["api.cu", "attn_pair.cu", "attn_tc.cu", "attn_simt.cu", "mask_kernel.cu", "pooled_pattern.cu", "vslash.cu",
           "api_decode.cu", "page_tables.cu", "qk_norm_rope.cu", "tree_attn.cu", "tree_attn_simt.cu"]
CALLS = os.path.join(HERE, "_decode_calls.so")
CALLS_SOURCE = os.path.join(CSRC, "decode_calls.cpp")
HEADERS = [os.path.join(CSRC, "common.cuh"), os.path.join(ROOT, "include", "shareprefill.h")]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS + [os.path.abspath(__file__)]
    extra = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    return any(os.path.getmtime(d) > t for d in deps + extra)


def _built_against() -> str | None:
    """What the Python entry is compiled against, as it is written into it; None without torch."""
    try:
        import torch
    except ImportError:
        return None
    return f"shareprefill calls for torch {torch.__version__}, Python {sysconfig.get_python_version()};"


def calls_match(path: str = CALLS) -> bool:
    """Whether the built Python entry is for the torch and the Python that run: it uses their C++ and C interfaces."""
    mark = _built_against()
    with open(path, "rb") as f:
        return mark is not None and mark.encode() in f.read()


def _start_calls_build():
    """Starts the compiler on the Python entry of the decode-side calls (half a minute: torch's headers); None without torch.
    The result goes to _new(CALLS)."""
    mark = _built_against()
    if mark is None:
        return None
    import torch
    from torch.utils import cpp_extension
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    nvcc = shutil.which(_nvcc())
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc))) if nvcc else "/usr/local/cuda"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DSP_BUILT_AGAINST="{mark}"', "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"),
           *[f"-I{p}" for p in cpp_extension.include_paths()], CALLS_SOURCE, "-o", _new(CALLS), "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    try:
        return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    except OSError as e:
        _no_calls(f"{e}\n")
        return None


def _new(path: str) -> str:
    return path[:-len(".so")] + ".new.so"


def _no_calls(out: str) -> None:
    """Without a working entry there is none: the decode-side calls then raise, and the library serves everything else."""
    if os.path.exists(CALLS):
        os.remove(CALLS)
    sys.stderr.write(out + "the compiler failed on decode_calls.cpp: the decode-side calls cannot be made from Python\n")


def _finish_calls_build(process) -> None:
    out, _ = process.communicate()
    if process.returncode == 0:
        os.replace(_new(CALLS), CALLS)
    else:
        _no_calls(out)


def calls_need_build() -> bool:
    if not os.path.exists(CALLS) or not calls_match(CALLS):
        return True
    t = os.path.getmtime(CALLS)
    return any(os.path.getmtime(d) > t for d in (CALLS_SOURCE, os.path.join(ROOT, "include", "shareprefill.h")))


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Builds the library (debug=True: the range-checked flavour, libshareprefill_debug.so, from the same sources), and
    beside it, where torch is installed, the Python entry of the decode-side calls."""
    lib = LIB_DEBUG if debug else LIB
    calls = _start_calls_build() if calls_need_build() or (force and not debug) else None
    try:
        if force or needs_build(lib):
            _build_library(lib, verbose, debug)
    finally:
        if calls is not None:
            _finish_calls_build(calls)
    return lib


def _build_library(lib: str, verbose: bool, debug: bool) -> None:
    objs = []
    procs = []
    for s in SOURCES:
        obj = os.path.join(CSRC, s.replace(".cu", ".dbg.o" if debug else ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, *(["-DSP_DEBUG"] if debug else []), "-c", os.path.join(CSRC, s), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for s, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {s}")
    link = [_nvcc(), "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", lib, *objs,
            "-cudart", "static", "-Xlinker", "--no-undefined", "-lpthread", "-ldl", "-lrt"]
    r = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout)
        raise RuntimeError("link failed")


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, debug="--debug" in sys.argv))
