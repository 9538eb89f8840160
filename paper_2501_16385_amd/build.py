"""Builds libfbq.so in-tree with hipcc for gfx950 (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OBJ_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libfbq.so")
CALL = os.path.join(HERE, "_fbq_call.so")     # the binding's call of fbq_linear: host code, a CPython module
SOURCES = ["fbq_api.cpp", "fbq_decode.hip", "fbq_decode_mfma.hip", "fbq_decode_stream.hip", "fbq_few_split.hip", "fbq_prefill.hip", "fbq_quantize.hip", "fbq_util.hip", "fbq_train.hip",
           "fbq_static.hip", "fbq_mix.hip",
           "fbq_cache.hip", "fbq_cache4.hip", "fbq_attend4_few.hip", "fbq_attend4_many.hip", "fbq_attend4_both.hip", "fbq_weigh.hip", "fbq_evict.hip",
           "fbq_attend_few.hip", "fbq_attend_many.hip", "fbq_attend_both.hip", "fbq_attention.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", INCLUDE, "-I", CSRC]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # the host pass does not know the gfx-only feature flag and says so once per file: harmless
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False, extra_flags=()) -> str:
    """Compiles every source (always, whatever is there already), the files side by side, and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    jobs = [[hipcc] + FLAGS + list(extra_flags) + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
    with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as pool:
        list(pool.map(lambda c: _run(c, verbose), jobs))
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs, verbose)
    _run([os.environ.get("CC", "gcc"), "-O2", "-std=c11", "-Wall", "-Wextra", "-fPIC", "-shared", "-I", INCLUDE, "-I", sysconfig.get_paths()["include"],
          os.path.join(CSRC, "fbq_call.c"), "-o", CALL], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
