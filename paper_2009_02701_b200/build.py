"""Build ``libhpsgd.so`` (CUDA, sm_100a only) in-tree with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhpsgd.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
# translation unit -> the headers it includes (beside those every unit has); each is compiled on its own
_COMMON = ["hpsgd_internal.h"]
_UNITS = {
    "hpsgd_api.cu": ["hpsgd_kernels.cuh", "hpsgd_state.cuh", "hpsgd_schedule.cuh", "hpsgd_staged.cuh"],
    "hpsgd_adamw.cu": ["hpsgd_ops_common.cuh"],
    "hpsgd_rmsnorm.cu": ["hpsgd_ops_common.cuh"],
    "hpsgd_quantize.cu": ["hpsgd_ops_common.cuh", "hpsgd_quantize.cuh"],
    "hpsgd_gemm.cu": ["hpsgd_ops_common.cuh", "hpsgd_tensor_core.cuh"],
    "hpsgd_scan.cu": ["hpsgd_ops_common.cuh"],
    "hpsgd_loss.cu": ["hpsgd_ops_common.cuh"],
    "hpsgd_ffn.cu": ["hpsgd_ops_common.cuh", "hpsgd_tensor_core.cuh", "hpsgd_quantize.cuh"],
}
SOURCES = [os.path.join(CSRC, u) for u in _UNITS]
# --fmad=false: the compiler never contracts a*b+c on its own; fused multiply-adds are
# written explicitly where the update rule has them.
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "--fmad=false", "-Xcompiler", "-fPIC", "-cudart", "static"]


def depends(unit: str) -> list:
    heads = [os.path.join(CSRC, h) for h in _COMMON + _UNITS[unit]]
    # this file too: it has the flags
    return [os.path.join(CSRC, unit), *heads, os.path.join(INCLUDE, "hpsgd.h"), os.path.join(INCLUDE, "hpsgd_ops.h"), os.path.abspath(__file__)]


DEPENDS = sorted({p for u in _UNITS for p in depends(u)})


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def build(force: bool = False, verbose: bool = False, debug: bool = False, out: str | None = None) -> str:
    """Compile the library if it is missing or older than its sources or than this file; returns its path.

    ``debug`` builds the checked variant (-DHPSGD_DEBUG: kernel guards that record and skip an
    out-of-range access, host-side validation of sparse row lists) into ``out`` (default
    ``libhpsgd_debug.so`` beside the normal library)."""
    lib = out or (os.path.join(HERE, "libhpsgd_debug.so") if debug else LIB)
    if not force and os.path.exists(lib):
        newest = max(os.path.getmtime(p) for p in DEPENDS)
        if os.path.getmtime(lib) >= newest:
            return lib
    objdir = os.path.join(HERE, "_build", "debug" if debug else "release")
    os.makedirs(objdir, exist_ok=True)

    def run(cmd):
        proc = subprocess.run(cmd, capture_output=True, text=True)
        if proc.returncode != 0:
            raise RuntimeError("nvcc failed:\n%s\n%s" % (proc.stdout, proc.stderr))
        if verbose:
            sys.stderr.write(proc.stderr)

    def compile_unit(unit):
        obj = os.path.join(objdir, unit[:-3] + ".o")
        if force or verbose or not os.path.exists(obj) or \
                os.path.getmtime(obj) < max(os.path.getmtime(p) for p in depends(unit)):
            tmp = obj + ".tmp.%d" % os.getpid()
            run([nvcc(), *NVCC_FLAGS, *(["-DHPSGD_DEBUG"] if debug else []), *(["-Xptxas", "-v"] if verbose else []),
                 "-c", "-o", tmp, os.path.join(CSRC, unit)])
            os.replace(tmp, obj)
        return obj

    with ThreadPoolExecutor(max_workers=len(_UNITS)) as pool:
        objects = list(pool.map(compile_unit, _UNITS))
    tmp = lib + ".tmp.%d" % os.getpid()
    run([nvcc(), *NVCC_FLAGS, "-shared", "-o", tmp, *objects])
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
