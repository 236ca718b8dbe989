"""Builds the HIP library (gfx950 only) in-tree with hipcc: libduo_verify.so (bf16 weights and KV cache) and
libduo_verify_fp16.so (the same sources compiled with DUO_FP16: IEEE fp16 instead)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libduo_verify.so")
LIB_PATH_FP16 = os.path.join(HERE, "libduo_verify_fp16.so")
CSRC = os.path.join(HERE, "csrc")
KERNEL_ORDER = os.path.join(HERE, "csrc", "kernel_order.txt")  # where the linker places the kernels, and why it matters
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument"]
# every source is a code object of its own; the list places the kernels of the first, the step's
SOURCES = {"duo_api.hip": ["-Xoffload-linker", "--symbol-ordering-file=" + KERNEL_ORDER], "duo_page.hip": [], "duo_scaled.hip": [], "duo_moe.hip": []}
TYPES = {LIB_PATH: [], LIB_PATH_FP16: ["-DDUO_FP16"]}


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "is not a recognized feature for this target" not in l)
    if verbose and out.strip():
        print(out, flush=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)


def build(verbose: bool = True) -> str:
    """Compiles both element types of every source (in parallel) and links the two libraries; returns the path of the bf16 library."""
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(max_workers=4) as pool:
        objects = {lib: [os.path.join(tmp, f"{os.path.basename(lib)}.{src}.o") for src in SOURCES] for lib in TYPES}
        jobs = [pool.submit(_run, [HIPCC, *FLAGS, *extra, *TYPES[lib], "-c", os.path.join(CSRC, src), "-o", obj], verbose)
                for lib in TYPES for (src, extra), obj in zip(SOURCES.items(), objects[lib])]
        for j in jobs:
            j.result()
        for lib in TYPES:
            _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objects[lib], "-o", lib], verbose)
    return LIB_PATH


if __name__ == "__main__":
    build()
    sys.exit(0)
