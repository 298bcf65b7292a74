"""Build the gfx950 HIP library (libpearl_attn.so) in-tree with hipcc.

Usage: python -m paper_2609_35158_amd.build   (or call build()).  Always recompiles."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libpearl_attn.so")
SOURCES = ["attn_kernels.hip", "decode_mx.hip", "kv_pages.hip", "kv_mx.hip", "rope.hip", "latent16.hip", "latent64.hip",
           "hbm_probe.hip", "api.cpp", "pd_engine.cpp"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # never form packed-fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # single-lane atomics stay plain: the atomic optimizer's wave reduction waits for the returned
    # value right away, which puts the atomics' latency on the kernels' critical paths
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


# Of some sources: the outputs of their matrix instructions stay in vector registers, where they are scaled; loops begin with a
# line of instructions (without it the main loop of latent64.hip is up to 1.5% slower, by what stands before it).
SOURCE_FLAGS = {s: ["-mllvm", "-amdgpu-mfma-vgpr-form", "-falign-loops=64"] for s in ("latent16.hip", "latent64.hip")}


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed (%d):\n%s" % (res.returncode, out))
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(max_workers=4) as pool:
        names = [os.path.join(objects, s + ".o") for s in SOURCES]
        jobs = [pool.submit(_run, [hipcc()] + HIPCC_FLAGS + SOURCE_FLAGS.get(s, []) +
                            ["-I", os.path.join(ROOT, "include"), "-c", "-o", o, os.path.join(CSRC, s)], verbose)
                for s, o in zip(SOURCES, names)]
        for j in jobs:
            j.result()
        _run([hipcc()] + HIPCC_FLAGS + ["-shared", "-o", tmp] + names, verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
