"""Builds libcapmoe.so (sm_100a only, nvcc) and the Python binding _bind.*.so (g++) in-tree.  `python -m paper_2503_05066_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libcapmoe.so")
BIND_SRC = os.path.join(CSRC, "bind.cpp")
SOURCES = ["api.cu", "route.cu", "drop.cu", "drop_cluster.cu", "drop_parallel.cu", "variants.cu", "permute_combine.cu", "ffn_simt.cu", "ffn_tc.cu", "ffn_tc_t.cu",
           "grouped_mm.cu", "grouped_fp8.cu", "gmm_rows.cu", "gmm_dw.cu", "gmm_swiglu8.cu",
           "norm.cu", "token_grad.cu", "route_grad.cu", "route_grad_tc.cu", "route_grad_any.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "nvcc"


def bind_path() -> str:
    """The binding's file for the running interpreter and torch: it is linked against both, so each pair has a file of its own."""
    import sysconfig
    import torch
    return os.path.join(PKG, f"_bind.{sysconfig.get_config_var('SOABI')}-torch-{torch.__version__}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}.so")


def _bind_cmd() -> list:
    """The binding against the running interpreter and torch, and the library beside it."""
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include"),
           sysconfig.get_paths()["include"]]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
            *[a for p in inc for a in ("-isystem", p)], BIND_SRC, "-o", bind_path(), "-L", PKG, "-l:libcapmoe.so", "-Wl,-rpath,$ORIGIN",
            "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"]


def _stale(obj: str, src: str) -> bool:
    if not os.path.exists(obj):
        return True
    newest = max(os.path.getmtime(p) for p in
                 [src, os.path.join(ROOT, "include", "capmoe.h"), __file__] +
                 [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")])
    return os.path.getmtime(obj) < newest


def build(force: bool = False, verbose: bool = False) -> str:
    header = os.path.join(ROOT, "include", "capmoe.h")
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))] + [header, __file__]
    fresh = lambda out, of: not force and os.path.exists(out) and os.path.getmtime(out) >= max(os.path.getmtime(p) for p in of)  # noqa: E731
    bound = fresh(bind_path(), [BIND_SRC, header, __file__])
    if fresh(LIB, deps) and bound:
        return LIB                       # up to date (object files need not exist: only the .so travel)
    objdir = os.path.join(PKG, "build")
    os.makedirs(objdir, exist_ok=True)
    nvcc = _nvcc()
    jobs = []
    for s in SOURCES:
        src, obj = os.path.join(CSRC, s), os.path.join(objdir, s.replace(".cu", ".o"))
        if force or _stale(obj, src):
            cmd = [nvcc, *NVCC_FLAGS, "-c", src, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)
    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
        return r.stderr
    if not fresh(LIB, deps):
        with ThreadPoolExecutor(max_workers=8) as ex:
            logs = list(ex.map(run, jobs))
        if verbose:
            print("\n".join(logs))
        run([nvcc, "-shared", "-o", LIB, *[os.path.join(objdir, s.replace(".cu", ".o")) for s in SOURCES], "-lcudart"])
    if not bound:
        run(_bind_cmd())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
