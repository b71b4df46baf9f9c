"""Builds ``libreader_verify.so`` (nvcc, sm_100a) and the Python module ``_marshal`` (g++) in-tree, without a GPU."""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(_HERE), "include")
LIB = os.path.join(_HERE, "libreader_verify.so")
MARSHAL = os.path.join(_HERE, "_marshal.so")   # csrc/marshal.cpp: torch tensors in, C ABI calls out
MARSHAL_MADE_FOR = os.path.join(CSRC, "_build", "marshal_made_for.txt")   # what it was compiled against, beside its source

SOURCES = ["api.cu", "tree_encode.cu", "verify_attn_generic.cu", "verify_attn_sm100.cu", "combine.cu",
           "accept.cu", "accept_noalloc.cu", "sample.cu", "kv_commit.cu", "kv_rearrange.cu", "padded_cache.cu", "accept_commit.cu",
           "rotate.cu", "prompt_attn_sm100.cu"]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall", "-I", INCLUDE, "-I", CSRC]


def _newest(files) -> float:
    return max(os.path.getmtime(f) for f in [os.path.join(INCLUDE, "reader_verify.h"), *files])


def _library_is_current() -> bool:
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]
    return os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest(files)


def _marshal_made_for() -> str:
    """What the module has to be compiled anew for: it is bound to this torch's C++ interface and this Python's."""
    import torch
    return f"torch {torch.__version__} at {os.path.dirname(torch.__file__)}, python {sys.version}"


def _marshal_is_current() -> bool:
    if not (os.path.exists(MARSHAL) and os.path.exists(MARSHAL_MADE_FOR)):
        return False
    with open(MARSHAL_MADE_FOR) as f:
        return f.read() == _marshal_made_for() and os.path.getmtime(MARSHAL) >= _newest([os.path.join(CSRC, "marshal.cpp")])


def _marshal_command(out: str) -> list:
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
            "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], "-isystem", "/usr/local/cuda/include",
            os.path.join(CSRC, "marshal.cpp"), "-o", out, "-L", lib, "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10_cuda", "-lc10",
            "-L", _HERE, "-l:libreader_verify.so", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{lib}"]


def _build_marshal(verbose: bool = False) -> None:
    tmp = MARSHAL + f".tmp{os.getpid()}"
    p = subprocess.run(_marshal_command(tmp), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if p.returncode != 0 or verbose:
        sys.stderr.write(f"--- marshal.cpp\n{p.stdout}\n")
    if p.returncode != 0:
        raise RuntimeError("g++ failed")
    os.replace(tmp, MARSHAL)
    os.makedirs(os.path.dirname(MARSHAL_MADE_FOR), exist_ok=True)
    with open(MARSHAL_MADE_FOR, "w") as f:
        f.write(_marshal_made_for())


def build(force: bool = False, verbose: bool = False) -> str:
    """The shared library, then the Python module that only the prompt calls need: what is missing or out of date of them."""
    if force or not _library_is_current():
        _build_library(verbose)
    if force or not _marshal_is_current():
        _build_marshal(verbose)
    return LIB


def _build_library(verbose: bool = False) -> None:
    """Compile every .cu into objects under csrc/_build and link the shared library."""
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    bdir = os.path.join(CSRC, "_build")
    os.makedirs(bdir, exist_ok=True)
    objs, procs = [], []
    extra = ["-Xptxas", "-v"] if verbose else []
    for s in SOURCES:
        o = os.path.join(bdir, s.replace(".cu", ".o"))
        objs.append(o)
        procs.append((s, subprocess.Popen([nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, s), "-o", o],
                                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for s, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- {s}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc, "-shared", "-o", tmp, *objs, "-lcudart"])
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
