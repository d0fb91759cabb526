"""Build libgdws.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import importlib.metadata
import os
import shutil
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
SOURCES = ["plan.cu", "plan_mem.cu", "f32.cu", "f32_tc.cu", "bf16.cu", "gdw_tc.cu", "pack.cu", "fused.cu", "fused_tc.cu", "fold.cu", "fold_split.cu", "api.cu", "static_ws.cu", "diag.cu", "rows.cu", "pointwise8.cu"]
HEADERS = [os.path.join(CSRC, "gdws_internal.h"), os.path.join(CSRC, "sm100.cuh"), os.path.join(CSRC, "rows.cuh"), os.path.join(_ROOT, "include", "gdws.h")]
LIB_PATH = os.path.join(_HERE, "libgdws.so")
BINDING = os.path.join(CSRC, "rows_binding.cpp")      # the calls on rows for Python, against torch's headers
BINDING_PATH = os.path.join(_HERE, "_rows.so")
BINDING_FOR = os.path.join(_HERE, "_build", "rows_binding.txt")      # the versions that it was built against

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
    "-Xcompiler", "-fPIC,-fvisibility=hidden", "--use_fast_math=false",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _torch_version():
    """The version of torch that the binding would be built against; None where there is no torch."""
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return None


def binding_is_stale() -> bool:
    """Whether ``_rows.so`` is missing, older than its sources, or built against another torch or Python, whose C++ interfaces it uses."""
    deps = [BINDING, os.path.join(_ROOT, "include", "gdws.h")]
    if not os.path.exists(BINDING_PATH) or any(os.path.getmtime(d) > os.path.getmtime(BINDING_PATH) for d in deps):
        return True
    try:
        with open(BINDING_FOR) as f:
            return f.read() != f"{_torch_version()} {sys.version}"
    except OSError:
        return True


def build_binding(force: bool = False) -> str:
    """Compile ``_rows.so`` (host code only, against torch's headers, by g++) next to this file; returns its path."""
    if not force and not binding_is_stale():
        return BINDING_PATH
    import sysconfig
    import torch
    home = os.path.dirname(torch.__file__)
    tmp = BINDING_PATH + f".tmp{os.getpid()}"
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                           "-I", os.path.join(_ROOT, "include"), "-isystem", os.path.join(home, "include"), "-isystem", os.path.join(home, "include", "torch", "csrc", "api", "include"),
                           "-isystem", sysconfig.get_paths()["include"], BINDING, "-o", tmp, "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, BINDING_PATH)
    os.makedirs(os.path.dirname(BINDING_FOR), exist_ok=True)
    with open(BINDING_FOR, "w") as f:
        f.write(f"{_torch_version()} {sys.version}")
    return BINDING_PATH


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile the CUDA sources into ``libgdws.so`` next to this file, and the binding of the calls on rows where there are torch and
    g++ (the library needs neither); returns the library's path."""
    if force or is_stale():
        _build_cuda(verbose)
    if _torch_version() and shutil.which("g++"):
        build_binding(force)
    return LIB_PATH


def _build_cuda(verbose: bool) -> None:
    objdir = os.path.join(_HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    nvcc = _nvcc()
    flags = [f for f in NVCC_FLAGS if f != "--use_fast_math=false"]
    if verbose:
        flags = flags + ["-Xptxas", "-v"]
    objs = []
    procs = []
    for s in SOURCES:
        o = os.path.join(objdir, s.replace(".cu", ".o"))
        cmd = [nvcc, *flags, "-I", os.path.join(_ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, s), "-o", o]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(o)
    for cmd, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode:
            sys.stderr.write(out)
        if pr.returncode:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    cmd = [nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp, *objs]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
