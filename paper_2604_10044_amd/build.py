"""Build liblg.so (HIP, gfx950) in-tree.

Every HIP source is compiled with hipcc for gfx950 only, with packed FP32 instructions disabled
(``-Xclang -target-feature -Xclang -packed-fp32-ops``; the host pass warns that it does not know
the feature, which is harmless), then linked into ``paper_2604_10044_amd/liblg.so``.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "liblg.so")
# (source, extra flags); lg_attend.hip is compiled in parts, in parallel
ATTEND_PARTS = 7
SOURCES = ([("lg_attend.hip", ("-DLG_ATTEND_PART=%d" % i,)) for i in range(ATTEND_PARTS)] +
           [(s, ()) for s in ("lg_detect.hip", "lg_prune.hip", "lg_capi.hip", "lg_copy.hip",
                            "lg_rope.hip", "lg_pages.hip", "lg_paged_attend.hip",
                            "lg_paged_capi.hip")])
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", INCLUDE, "-I", CSRC]


def _compile(unit) -> str:
    src, extra = unit
    part = "".join("_" + f.rsplit("=", 1)[-1] for f in extra)
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + part + ".o")
    cmd = [HIPCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source (always) and link liblg.so; returns the library path."""
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
