"""Builds libecrm.so (gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libecrm.so")
SOURCES = ["ecrm_api.hip", "sort.hip", "update.hip", "chains.hip", "buckets.hip", "direct.hip", "recover.hip", "reads.hip", "holdback.hip", "probe.hip",
           "embed.hip", "token_sort.hip", "embed_grad.hip", "grads.hip", "dropout.hip", "ffn.hip", "ffn_plan.hip",
           "ffn_bf16.hip", "ffn_f16.hip", "ffn_f32.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-result"]


def build(verbose: bool = False, out: str = LIB, defines=()) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_ = [hipcc, *FLAGS, *[f"-D{d}" for d in defines], "-I", os.path.join(ROOT, "include"), "-I", CSRC]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    # the sources side by side, the ones that take longest first
    with tempfile.TemporaryDirectory() as objects:
        sources = sorted(SOURCES, key=lambda s: not s.startswith("ffn_"))
        made = [os.path.join(objects, os.path.splitext(s)[0] + ".o") for s in sources]
        with ThreadPoolExecutor(int(os.environ.get("MAX_JOBS") or min(8, os.cpu_count() or 1))) as pool:
            list(pool.map(lambda s, o: run([*compile_, "-c", os.path.join(CSRC, s), "-o", o]), sources, made))
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *made, "-o", out])
    return out


if __name__ == "__main__":
    print(build(verbose=True))
