"""Builds the gfx950 shared library ``libsp_amd.so`` in-tree with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libsp_amd.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]
# device code that is given no NaNs and produces none on purpose: lets fmaxf chains become v_max3_f32 without
# canonicalising moves (host-side argument checks keep full NaN semantics)
NO_NANS = ["-Xarch_device", "-fno-honor-nans"]
# ... but for what may meet them and has to let them through: the cache stores what it is given, and attention makes
# a row NaN that sees one. With the flag a NaN there would mean nothing to the compiler.
HONOUR_NANS = {"sp_cache.hip", "sp_attend.hip", "sp_weights.hip", "sp_evict.hip", "sp_mx4.hip"}


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def compile_command(src: str, obj: str):
    flags = FLAGS + ([] if os.path.basename(src) in HONOUR_NANS else NO_NANS)
    return [HIPCC, *flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj]


def link_command(objs):
    return [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH, *objs]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out, flush=True)


def build_library(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory() as tmp:
        pairs = [(s, os.path.join(tmp, os.path.basename(s) + ".o")) for s in sources()]
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda p: _run(compile_command(*p), verbose), pairs))
        _run(link_command([o for _, o in pairs]), verbose)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
    sys.exit(0)
