"""Build libasgd.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

Each source compiles to an object under ``_build/`` (in parallel), then one
shared library is linked next to this file.  Every call rebuilds.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libasgd.so")
BUILD_DIR = os.path.join(ROOT, "_build")
ARCH = "gfx950"

# hipcc options: no packed-fp32 instructions (v_pk_*_f32) anywhere in device code.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Wall",
          "-Wno-unused-result", "-I", os.path.join(ROOT, "include")]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found; the HIP library cannot be built")


def sources() -> list:
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")) +
                  glob.glob(os.path.join(PKG, "csrc", "*.cpp")))


# Per-source options.  k_out_bwd.hip: matrix instructions write their results to
# ordinary vector registers, so that the exponentials read the recomputed logits and
# the W2 update reads dW2 without first copying them out of accumulation registers
# (a kernel with the whole register file would otherwise get the accumulation form;
# the operands pinned to accumulation registers stay there).  k_label_narrow.hip: the
# same for its logits, which the softmax reads at once.
FILE_FLAGS = {f: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for f in ("k_out_bwd.hip", "k_label_narrow.hip")}


def _compile(src: str, extra: list, verbose: bool) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = ([hipcc()] + COMMON + DEVICE_FLAGS + FILE_FLAGS.get(os.path.basename(src), []) + extra +
           ["-c", src, "-o", obj])
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return obj


def build(verbose: bool = False, extra: list = ()) -> str:
    """Compile every source and link ``libasgd.so``; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sources()
    jobs = min(len(srcs), max(1, min(8, os.cpu_count() or 1)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, list(extra), verbose), srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv,
                extra=["-Rpass-analysis=kernel-resource-usage"] if "--resources" in sys.argv else []))
