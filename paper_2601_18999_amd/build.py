"""Build libkvr.so (HIP, gfx950) in-tree with hipcc.

Usage: ``python -m paper_2601_18999_amd.build``.  The library is plain
HIP + C++ behind the C ABI of include/kvr.h; it does not link against torch.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libkvr.so")
# the simulator, and the serving operators
SOURCES = ["csrc/kvr_device.hip", "csrc/kvr_api.cpp", "csrc_serve/kvr_serve.hip", "csrc_serve/kvr_serve_api.cpp",
           "csrc_serve/kvr_attend_64.hip", "csrc_serve/kvr_attend_128.hip", "csrc_serve/kvr_attend_256.hip",
           "csrc_serve/kvr_layer_api.cpp", "csrc_serve/kvr_norm.hip", "csrc_serve/kvr_product.hip",
           "csrc_serve/kvr_linear.hip"]
ARCH = os.environ.get("KVR_OFFLOAD_ARCH", "gfx950")

FLAGS = [
    "-O3", "-std=c++17", "-fPIC",
    # no fused multiply-add: results must equal the IEEE left-to-right definition
    "-ffp-contract=off",
    # keep packed fp32 instructions out of the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # atomics stay single instructions: nearly all are one lane's, and the wave
    # reduction that the optimiser puts around them costs the step kernel 2 to 4%
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
]
# of single sources: in the attention kernels scalar registers are short, and
# this scheduler counts them (without it they spill into the inner loop: 924
# against 804 us for 9,216 new tokens of 32 heads).  Their assembler names M0 as
# written, which the compiler would remark upon for each statement.
EXTRA = {f"csrc_serve/kvr_attend_{d}.hip": ["-mllvm", "-amdgpu-use-amdgpu-trackers=1", "-Wno-inline-asm"]
         for d in (64, 128, 256)}
EXTRA["csrc_serve/kvr_product.hip"] = ["-Wno-inline-asm"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False) -> str:
    """Compile every source (side by side) and link libkvr.so (always recompiles)."""
    tmp = LIB + ".tmp"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    with tempfile.TemporaryDirectory() as tdir, ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:
        objects = [os.path.join(tdir, os.path.splitext(os.path.basename(s))[0] + ".o") for s in SOURCES]
        list(pool.map(run, [[hipcc(), f"--offload-arch={ARCH}", *FLAGS, *EXTRA.get(s, []), "-c", "-o", o,
                             os.path.join(HERE, s)]
                            for s, o in zip(SOURCES, objects)]))
        run([hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", "-o", tmp, *objects])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
