"""Build liblora_cache.so (host code + gfx950 kernels) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblora_cache.so")

SOURCES = ["lora_cache.cpp", "indexer.cpp", "scheduler.cpp", "gemv_kernels.hip", "mfma_kernels.hip", "linear_kernels.hip", "fill_kernels.hip",
           "kv_cache.cpp", "kv_kernels.hip", "attn_kernels.hip", "attn_e4m3_kernels.hip"]

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-munsafe-fp-atomics",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the leading scalar arguments of a kernel arrive in registers with the wavefront
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False) -> str:
    """Every source is compiled each time, several at once, and the objects are linked."""
    flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp:
        def compile_one(name: str):
            obj = os.path.join(tmp, name + ".o")
            cmd = [hipcc(), *flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "-c", os.path.join(CSRC, name), "-o", obj]
            return obj, cmd, subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)

        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1, 8)) as pool:
            done = list(pool.map(compile_one, SOURCES))
        link = [hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", *[obj for obj, _cmd, _res in done], "-o", LIB]
        steps = [(cmd, res) for _obj, cmd, res in done]
        if all(res.returncode == 0 for _cmd, res in steps):
            steps.append((link, subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, res in steps:
        out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
        if verbose:
            print(" ".join(cmd), flush=True)
        if res.returncode != 0:
            sys.stderr.write(out + "\n")
            raise RuntimeError("hipcc failed building liblora_cache.so")
        if verbose and out.strip():
            print(out)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
