"""Build libfarskip.so for gfx950 with hipcc (in-tree, no JIT cache).

    python -m paper_2511_11505_amd.build
"""

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libfarskip.so")
ARCH = os.environ.get("FS_OFFLOAD_ARCH", "gfx950")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

COMMON = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-result",
    # packed fp32 vector ops stay off on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(HERE, "..", "include"),
]
# The router's fixed fp32 reduction order needs products and sums rounded
# separately for fp32 inputs: no contraction in that file.
PER_FILE = {"router.hip": ["-ffp-contract=off"]}
SOURCES = ["api.cpp", "router.hip", "dispatch.hip", "gemm.hip", "gemm_r64.hip", "gemm_r192_gateup.hip", "gemm_r192_down.hip",
           "gemm_r192_fp8.hip", "elementwise.hip", "fp8.hip",
           "standin.hip", "api_layer.cpp", "linear.hip", "linear_any.hip", "linear_few.hip", "linear_mid.hip", "linear_tile_fwd.hip",
           "linear_tile_da.hip", "linear_tile_dw.hip", "norm.hip", "checkpoint.hip",
           "api_attention.cpp", "rotary.hip", "attention.hip", "attention_bf16.hip", "attention_codes.hip",
           "attention_f32.hip", "attention_codes_f32.hip"]


def _compile(src):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *COMMON, *PER_FILE.get(src, []), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {src}\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj, r.stderr


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        results = list(ex.map(_compile, SOURCES))
    if verbose:
        for obj, err in results:
            if err.strip():
                print(err, file=sys.stderr)
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *[o for o, _ in results]]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
