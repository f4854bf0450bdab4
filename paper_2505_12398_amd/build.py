"""Build libtv.so (the HIP kernels and the C-ABI) in-tree for gfx950."""

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libtv.so")

SOURCES = ["tv_abi.cpp", "tv_ops_abi.cpp", "tv_kernels.hip", "tv_commit.hip", "tv_lmhead.hip",
           "tv_logits.hip", "tv_cache.hip", "tv_fp4.hip", "tv_attention.hip",
           "tv_attention_fp4.hip", "tv_prompt.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed fp32 instructions (v_pk_*_f32) in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]

# The prompts' kernel holds 490 registers of a wavefront's 512: its products' results that the vector
# unit reads in those that it can read, the rest in the others (by itself the compiler puts all results
# into those, and copies 60 a step).
SOURCE_FLAGS = {"tv_prompt.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def build(verbose: bool = False) -> str:
    """Compile every source into paper_2505_12398_amd/libtv.so; returns its path."""
    tmp = LIB + ".tmp"
    compile_flags = [f for f in FLAGS if f != "-shared"]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as out:
        objects = [os.path.join(out, s + ".o") for s in SOURCES]
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: run([HIPCC, *compile_flags, *SOURCE_FLAGS.get(so[0], []),
                                          "-I", INCLUDE, "-I", CSRC, "-c",
                                          os.path.join(CSRC, so[0]), "-o", so[1]]),
                          zip(SOURCES, objects)))
        run([HIPCC, "--offload-arch=gfx950", "-shared", *objects, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
