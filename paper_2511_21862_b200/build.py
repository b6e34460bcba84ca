"""Compile the CUDA sources into `libooco.so` and the call marshalling of `spec` into `_spec_calls.so`, next to this file
(sm_100a only, in-tree)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libooco.so")
LIB_CHECKED = os.path.join(HERE, "libooco_checked.so")   # the same sources with -DOOCO_CHECKS
SOURCES = ["ooco_api.cu", "ooco_spec.cu", "ooco_batch.cu", "ooco_chunk.cu", "ooco_sched.cpp"]
HEADERS = ["decode_kernels.cuh", "chunk_kernels.cuh", "chunk_tc_kernels.cuh", "chunk_tc2_kernels.cuh", "block_copy_kernels.cuh", "tree_kernels.cuh", "spec_kernels.cuh", "cta_util.cuh", "norm_rope_kernels.cuh",
           "page_kernels.cuh", "logits_kernels.cuh", "packed_kernels.cuh", "api_internal.h", "ptx.cuh", os.path.join("..", "..", "include", "ooco.h"),
           os.path.join("..", "..", "include", "ooco_spec.h"), os.path.join("..", "..", "include", "ooco_batch.h"),
           os.path.join("..", "..", "include", "ooco_sched.h")]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "--expt-relaxed-constexpr", "-t", "0"]


CALLS = os.path.join(HERE, "_spec_calls.so")             # CPython module, host code only
CALLS_SOURCES = ["py_spec.cpp", "py_batch.cpp"]
CALLS_HEADERS = ["py_calls.h"] + [os.path.join("..", "..", "include", f) for f in ("ooco.h", "ooco_spec.h", "ooco_batch.h")]


def _built_for() -> str:
    """What the marshalling module is tied to beside its sources: it uses torch's and the interpreter's binary interfaces."""
    import torch
    return f"torch {torch.__version__} python {sys.version_info[0]}.{sys.version_info[1]}"


def is_stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    files = CALLS_SOURCES + CALLS_HEADERS if lib == CALLS else SOURCES + HEADERS
    deps = [os.path.join(CSRC, f) for f in files] + [os.path.abspath(__file__)]
    if any(os.path.getmtime(d) > t for d in deps if os.path.exists(d)):
        return True
    if lib != CALLS:
        return False
    with open(lib, "rb") as f:   # (the module carries the text, see py_spec.cpp)
        return _built_for().encode() + b"\0" not in f.read()


def build_calls(force: bool = False) -> str:
    """Run the C++ compiler on the marshalling module if it is missing, older than its sources or built for another torch."""
    if force or is_stale(CALLS):
        import torch
        from torch.utils.cpp_extension import include_paths, library_paths
        # (the system's compiler: it shares the C++ runtime that torch and the interpreter use)
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-DNDEBUG", f'-DOOCO_BUILT_FOR="{_built_for()}"',
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
               *[f"-I{p}" for p in include_paths("cuda") + [sysconfig.get_path("include")]], "-o", CALLS,
               *[os.path.join(CSRC, f) for f in CALLS_SOURCES], *[f"-L{p}" for p in library_paths()],
               "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError(f"the C++ compiler failed building {os.path.basename(CALLS)}")
    return CALLS


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Run nvcc if the library is missing or older than its sources; returns the library path.
    `checked`: the variant whose kernels range-check every device-derived index (libooco_checked.so)."""
    lib = LIB_CHECKED if checked else LIB
    if force or is_stale(lib):
        nvcc = os.environ.get("NVCC", "nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-DOOCO_CHECKS"] if checked else []) + (["-Xptxas", "-v"] if verbose else []) + \
              ["-o", lib] + [os.path.join(CSRC, f) for f in SOURCES]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed building {os.path.basename(lib)}")
    if not checked:
        try:
            build_calls(force)
        except (RuntimeError, OSError, ImportError) as e:
            # The C ABI and `binding` need neither a C++ compiler nor Python's and torch's headers: only `spec` goes without.
            if os.path.exists(CALLS):
                os.remove(CALLS)   # (a module of older sources, or of another torch, must not be loaded)
            sys.stderr.write(f"{os.path.basename(CALLS)} could not be built ({e}): {os.path.basename(lib)} is complete, but "
                             "paper_2511_21862_b200.spec cannot be used\n")
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
