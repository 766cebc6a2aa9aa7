"""Builds libdartquant.so (sm_100a only, nvcc) and the module _calls (its Python calls, the host compiler) in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libdartquant.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))   # of this interpreter
UNTAGGED = os.path.join(HERE, "_calls.so")                                       # any interpreter would load it
OBJ_DIR = os.path.join(HERE, "_build")
SOURCES = ["api.cu", "gemm_ffma.cu", "qr_forward.cu", "qr_backward.cu", "tc_path.cu", "qr_tc.cu", "qr_panel_tc.cu", "qr128.cu", "token_sampling.cu", "eval_metrics.cu", "cayley_tc.cu", "objectives.cu", "qr128_inc.cu", "qr128_tc5.cu", "mx_quant.cu", "mx_matmul.cu", "mx_api.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _stale() -> bool:
    if not (os.path.exists(LIB) and os.path.exists(CALLS)):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "dartquant.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
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
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"],
                        "-I", INCLUDE, os.path.join(CSRC, "py_calls.cpp"), "-o", CALLS], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("host compiler failed for py_calls.cpp:\n" + r.stderr)
    if os.path.exists(UNTAGGED):
        os.remove(UNTAGGED)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
