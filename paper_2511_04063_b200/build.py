"""Builds libdartquant.so (sm_100a only, nvcc) and the module _calls (its Python calls, the host compiler) in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libdartquant.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))   # of this interpreter
UNTAGGED = os.path.join(HERE, "_calls.so")                                       # any interpreter would load it
OBJ_DIR = os.path.join(HERE, "_build")
SOURCES = ["api.cu", "gemm_ffma.cu", "qr_forward.cu", "qr_backward.cu", "tc_path.cu", "qr_tc.cu", "qr_panel_tc.cu", "qr128.cu", "token_sampling.cu", "eval_metrics.cu", "cayley_tc.cu", "objectives.cu", "qr128_inc.cu", "qr128_tc5.cu", "mx_quant.cu", "mx_matmul.cu", "mx_api.cu", "qk_rope.cu", "kv_cache.cu", "kv_attention.cu", "kv_prompt.cu", "kv_api.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps: list[str]) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(p) > os.path.getmtime(target) for p in deps)


def _build_library(verbose: bool) -> None:
    os.makedirs(OBJ_DIR, exist_ok=True)
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(OBJ_DIR, src.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s" % (src, r.stderr))
        if verbose and r.stderr:
            print(r.stderr, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    r = subprocess.run([nvcc, "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a"],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)


def _build_calls(source: str) -> None:
    """The Python calls of the microscaled operators; the only part that needs Python's headers."""
    include = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(include, "Python.h")):
        warnings.warn("no Python.h in %s: the microscaled operators have no Python calls; everything else is built" % include)
        return
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-I", include,
                        "-I", INCLUDE, source, "-o", CALLS], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("host compiler failed for py_calls.cpp:\n" + r.stderr)


def build(force: bool = False, verbose: bool = False) -> str:
    header, calls = os.path.join(INCLUDE, "dartquant.h"), os.path.join(CSRC, "py_calls.cpp")
    if force or _stale(LIB, [header, *(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "py_calls.cpp")]):
        _build_library(verbose)
    if force or _stale(CALLS, [header, calls]):
        _build_calls(calls)
    if os.path.exists(UNTAGGED):
        os.remove(UNTAGGED)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
