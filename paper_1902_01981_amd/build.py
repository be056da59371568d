"""Builds libcodedreduce.so (host plan + C-ABI + gfx950 kernels) and libcodedreduce_layers.so (layers of networks) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcodedreduce.so")
SOURCES = ["gc_design.cpp", "tree_plan.cpp", "latency_model.cpp", "codedreduce.cpp", "kernels.hip"]
LAYERS_LIB = os.path.join(HERE, "libcodedreduce_layers.so")
LAYERS_SOURCES = ["layers.cpp", "norm_rows.hip", "norm_forward.hip", "norm_backward.hip", "dropout_kernels.hip", "loss_kernels.hip",
                  "embedding_kernels.hip", "log_probs_kernels.hip", "distill_kernels.hip"]
# the packed-fp32 target feature is switched off for all device code
DEVICE_FLAGS = ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose: bool = False) -> str:
    _library(LAYERS_LIB, LAYERS_SOURCES, verbose)
    return _library(LIB, SOURCES, verbose)


def _library(lib: str, sources, verbose: bool) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(bdir, src + ".o")
        cmd = [hipcc, "-O3", "-std=c++17", "-fPIC", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
        if src.endswith(".hip"):
            cmd += DEVICE_FLAGS
        else:
            cmd += ["-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")]
        cmd += ["-c", os.path.join(CSRC, src), "-o", obj]
        _run(cmd, verbose)
        return obj

    with ThreadPoolExecutor(max_workers=4) as pool:          # a compiler each
        objs = list(pool.map(compile_one, sources))
    # the interface and nothing else: helpers with plain names would meet a program's own
    _run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-Wl,--version-script=" + os.path.join(CSRC, "exports.map"), "-o", lib] + objs, verbose)
    return lib


def _run(cmd, verbose):
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if verbose or res.returncode != 0:
        sys.stderr.write(" ".join(cmd) + "\n" + res.stdout + err + "\n")
    if res.returncode != 0:
        raise RuntimeError("build failed: " + " ".join(cmd))


if __name__ == "__main__":
    print(build(verbose=True))
