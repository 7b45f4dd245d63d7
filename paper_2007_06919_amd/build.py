"""Build ``libaqd.so`` (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

Every source is compiled on each call (the build check compiles even when a
library exists); objects go to ``_build/`` and the shared library next to
this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libaqd.so")
SOURCES = ["aqd_api.hip", "qconv_mfma.hip", "qconv_wv.hip", "qconv_wvs.hip", "qconv_b8.hip", "qconv_gf.hip", "qconv_fx.hip", "qconv_stem.hip", "qconv_splitk.hip", "qconv_direct.hip",
           "qadd.hip", "qpool.hip", "qrows.hip", "qlin.hip", "qlin_f32.hip", "qlin_f16.hip", "qlin_bf16.hip",
           "heads.hip", "qcache.hip", "qattn.hip", "attn.hip", "mfma_probe.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    "-ffp-contract=off",                      # host parameter derivation: IEEE, no FMA
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-command-line-argument",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]
# the attention's vector units read and write what its matrix cores do: accumulators stay in vector registers as long as they fit
FILE_FLAGS = {"attn.hip": ("-mllvm", "-amdgpu-mfma-vgpr-form=1")}


def _compile(src: str, verbose: bool, extra) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *FILE_FLAGS.get(src, ()), *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if verbose and r.stderr.strip():
        print(r.stderr, flush=True)
    return obj


def build(verbose: bool = False, extra=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose, list(extra)), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    extra = ["-Rpass-analysis=kernel-resource-usage"] if "--resource-usage" in sys.argv else []
    print(build(verbose="-v" in sys.argv or bool(extra), extra=extra))
