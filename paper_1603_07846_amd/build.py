"""Build the gfx950 HIP library ``libsinga_mi.so`` in-tree.

Every source is compiled with hipcc for gfx950 only and linked into one
shared library next to this file.  Packed-fp32 instruction forms are disabled
(``-target-feature -packed-fp32-ops``); the kernels never need them.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_NAME = "libsinga_mi.so"
LIB_PATH = os.path.join(HERE, LIB_NAME)
SOURCES = ["abi.cpp", "noalloc.cpp", "trace.cpp", "conv_igemm.hip", "conv_fwd_tile.hip", "conv_wgrad_tile.hip", "conv_aux.hip", "eltwise.hip",
           "dense_abi.cpp", "dense_bf16.hip", "dense_f32.hip", "dense_aux.hip", "gradnorm.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"


def _flags(tuning=False):
    # tuning: a measurement build whose dispatch reads the SINGA_* layout and
    # split overrides from the environment (the default build ignores them)
    return (["-DSINGA_TUNING"] if tuning else []) + ["-O3", "-std=c++17", "-fPIC", "--offload-arch=" + ARCH, "-I", INCLUDE, "-I", CSRC,
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-Wno-unused-command-line-argument"]


def build(verbose: bool = False, tuning: bool = False) -> str:
    """Compile all sources (always) and link the library; returns its path."""
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        cmd = [HIPCC] + _flags(tuning) + lang + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        # the host pass does not know the packed-fp32 feature; that warning is harmless
        text = "\n".join(l for l in text.splitlines() if "packed-fp32-ops" not in l)
        if text.strip() and (verbose or p.returncode):
            print(text, file=sys.stderr)
        if p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError("hipcc failed for: " + ", ".join(failed))
    tmp = LIB_PATH + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "-shared", "-fPIC", "--offload-arch=" + ARCH, "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, tuning="--tuning" in sys.argv))
