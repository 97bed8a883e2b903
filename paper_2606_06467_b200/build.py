"""Build libclsa.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the CPython module that marshals some calls."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libclsa.so")
MARSHAL = os.path.join(PKG, "_marshal" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))  # CPython module (csrc/marshal.c)
SOURCES = ["api.cu", "index_scores.cu", "index_gemm.cu", "index_topk.cu", "topk.cu", "topk_filter.cu", "sparse_attn.cu", "sparse_attn_sk.cu", "project_append.cu",
           "api_cache8.cu", "norm_rope.cu", "cache8_append.cu", "index_scores8.cu", "sparse_attn8.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers += [os.path.join(ROOT, "include", f) for f in ("clsa.h", "clsa_cache8.h")]
    objdir = os.path.join(PKG, "build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(objdir, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode != 0:
            sys.stderr.write(out)
        if pr.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    if force or procs or _stale(LIB, objs):
        tmp = LIB + f".{os.getpid()}.tmp"
        subprocess.check_call([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp] + objs
                              + ["-Xcompiler", "-fPIC"])
        os.replace(tmp, LIB)
    src = os.path.join(CSRC, "marshal.c")
    include = sysconfig.get_paths()["include"]
    if os.path.exists(os.path.join(include, "Python.h")) and (force or _stale(MARSHAL, [src] + headers)):
        tmp = MARSHAL + f".{os.getpid()}.tmp"
        subprocess.check_call(["gcc", "-O2", "-std=c11", "-Wall", "-Wno-cast-function-type", "-fPIC", "-shared", "-I", include,
                               "-I", os.path.join(ROOT, "include"), "-o", tmp, src])
        os.replace(tmp, MARSHAL)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
