"""Compiles libgdn.so (the HIP kernels and the C ABI) for gfx950 with hipcc, in-tree."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libgdn.so")
SOURCES = [os.path.join(CSRC, f) for f in ("gdn_api.hip", "gdn_ops_api.hip", "gdn_block_api.hip")]
HEADERS = [os.path.join(CSRC, f) for f in ("gdn_act.h", "gdn_backward.h", "gdn_clip.h", "gdn_conv.h",
                                           "gdn_device.h", "gdn_frame.h", "gdn_gated.h", "gdn_gated_rule.h", "gdn_host.h",
                                           "gdn_kernels.h", "gdn_norm.h", "gdn_step.h")] + \
          [os.path.join(INCLUDE, f) for f in ("gdn.h", "gdn_block.h", "gdn_ops.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed fp32 VALU instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


# MFMA accumulators in ordinary VGPRs: avoids AGPR<->VGPR copies whenever
# VALU code touches an accumulator (state scaling, bf16 conversion).  The tiled products of
# gdn_block_api.hip only accumulate, and choose for themselves.
VGPR_FORM = ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]


def build(verbose: bool = False, extra_flags=()) -> str:
    """Every source to an object of its own, at the same time, then one link."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f != "-shared"] + list(extra_flags)
    jobs = [(src, os.path.splitext(src)[0] + ".o") for src in SOURCES]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with ThreadPoolExecutor(len(jobs)) as pool:
        list(pool.map(lambda j: run([hipcc, *flags, *([] if "gdn_block_api" in j[0] else VGPR_FORM), "-I", INCLUDE, "-I", CSRC, "-c", "-o", j[1], j[0]]), jobs))
    run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB + ".tmp", *(o for _, o in jobs)])
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
