"""Builds libqvg.so (the C-ABI library) for gfx950 with hipcc, in-tree.

hipcc cross-compiles without a GPU.  Flags that matter for correctness:
-ffp-contract=off (no multiply-add fusion except where fmaf is written: the stored
2-bit codes depend on single IEEE operations), correctly rounded fp32 division, and
packed-fp32 code generation switched off.
"""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqvg.so")
SOURCES = ["qvg_api.cpp", "qvg_decode.hip", "qvg_encode.hip", "qvg_lloyd.hip", "qvg_kmeans.hip", "qvg_quant.hip", "qvg_attn.hip", "qvg_attn_slab.hip",
           "qvg_tree.hip", "qvg_tree_packed.hip", "qvg_tree_wide.hip", "qvg_pages.hip", "qvg_rope.hip", "qvg_attn_pages.hip"]
HEADERS = [os.path.join(CSRC, "qvg_internal.hpp"), os.path.join(CSRC, "qvg_attn_tiles.hpp"), os.path.join(CSRC, "qvg_tree.hpp"), os.path.join(CSRC, "qvg_rows.hpp"), os.path.join(CSRC, "qvg_attn_pages.hpp"), os.path.join(CSRC, "qvg_tree_lane.hpp"), os.path.join(CSRC, "qvg_kmeans.hpp"), os.path.join(CSRC, "qvg_assign.hpp"),
           os.path.join(ROOT, "include", "qvg.h")]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
    "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = True, verbose: bool = False, extra_flags=()) -> str:
    """Compile every source and link libqvg.so.  Returns its path."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(objdir, src + ".o")
        objs.append(obj)
        cmd = [hipcc, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd))
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    for src, pr in procs:
        out, _ = pr.communicate()
        text = out.decode(errors="replace")
        # the host pass does not know the packed-fp32 feature name: harmless
        text = "\n".join(l for l in text.splitlines() if "packed-fp32-ops" not in l)
        if pr.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{text}")
        if verbose and text.strip():
            print(text)
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], check=True)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
