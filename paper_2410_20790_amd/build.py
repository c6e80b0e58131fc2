"""Build libsparsetem.so (HIP for gfx950) in the package directory.

Usage: python -m paper_2410_20790_amd.build
"""

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")          # the encoder
OPS = os.path.join(PKG, "csrc_ops")      # the operators behind it
OUT = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libsparsetem.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", OPS]
# Packed-FP32 instructions are disabled for all device code.
DEVICE = ["-x", "hip", f"--offload-arch={ARCH}", "-Xclang", "-target-feature",
          "-Xclang", "-packed-fp32-ops", "-munsafe-fp-atomics"]
# The operators fuse a product and a sum where their source says so: a step
# taken alone and in a chunk, by another kernel, has the same bits.
EXACT = DEVICE + ["-ffp-contract=off"]

SOURCES = [
    ("st_plan.cpp", []),
    ("st_kernels.hip", DEVICE),
    ("st_dense.hip", DEVICE),
    ("st_gather.hip", DEVICE),
    ("st_exec.hip", DEVICE),
    ("../csrc_ops/norm.hip", EXACT),
    ("../csrc_ops/norm_grad.hip", EXACT),
    ("../csrc_ops/time_conv.hip", EXACT),
    ("../csrc_ops/time_conv_grad.hip", EXACT),
    ("../csrc_ops/gated_scan.hip", EXACT),
    ("../csrc_ops/gated_scan_grad.hip", EXACT),
]


def _compile(src, extra):
    name = os.path.splitext(os.path.basename(src))[0]
    obj = os.path.join(OUT, name + ".o")
    cmd = [HIPCC, *extra, *COMMON, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n"
                           f"{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(OUT, exist_ok=True)
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        objs = list(ex.map(lambda a: _compile(*a), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o",
           tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
