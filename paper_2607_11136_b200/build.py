"""Builds the CUDA library in-tree, paper_2607_11136_b200/libxema.so (sm_100a only), and the module that calls its
feed-forward operators with torch tensors, paper_2607_11136_b200/_torch_ops.so."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor
from importlib import metadata, util

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libxema.so")

TORCH_OPS = os.path.join(HERE, "_torch_ops.so")

SOURCES = ["planner.cpp", "elementwise.cu", "gemm.cu", "attention.cu", "rms_norm.cu", "gated_ffn.cu", "lora.cu", "runtime.cu", "static_arena.cu", "selftest.cu", "pluggable.cpp"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def _stale(target: str, deps: list) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_ops_command(source: str) -> list:
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi()]
            + ["-I" + p for p in include] + [source, "-o", TORCH_OPS, "-L" + os.path.join(root, "lib")]
            + ["-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_python"])


def _torch_stamp() -> str:
    """The torch and the Python that the module for torch tensors is built against."""
    return "torch %s at %s, Python %s\n" % (metadata.version("torch"), util.find_spec("torch").origin, sys.version)


def _read(path: str) -> str:
    if not os.path.exists(path):
        return ""
    with open(path) as f:
        return f.read()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every source for sm_100a and links libxema.so and _torch_ops.so.  Returns the library path."""
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(os.path.dirname(HERE), "include", "xema.h"))
    nvcc = _nvcc()
    jobs = []
    objs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
        objs.append(o)
        if force or _stale(o, [s] + headers):
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            jobs.append(cmd)

    torch_ops = os.path.join(CSRC, "torch_ops.cpp")
    links = len(jobs)
    stamp = os.path.join(OBJ, "torch_ops.stamp")
    if force or _stale(TORCH_OPS, [torch_ops, headers[-1]]) or _read(stamp) != _torch_stamp():
        jobs.append(_torch_ops_command(torch_ops))

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("build failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
        return r.stderr

    with ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 1))) as ex:
        for out in ex.map(run, jobs):
            if verbose and out:
                print(out, file=sys.stderr)
    if len(jobs) > links:
        with open(stamp, "w") as f:
            f.write(_torch_stamp())
    if links or force or _stale(LIB, objs):
        run([nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
