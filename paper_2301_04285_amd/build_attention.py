"""Builds the C-ABI shared library ``libtaps_attention.so`` for gfx950 with hipcc.

Run as ``python -m paper_2301_04285_amd.build_attention``; the library lands
next to this file so that it travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys

from .build import ARCH, CSRC, HERE, INCLUDE, hipcc

LIB = os.path.join(HERE, "libtaps_attention.so")
SOURCES = ["taps_attention_api.hip", "taps_norm_rotate.hip", "taps_attend.hip", "taps_mx_api.hip",
           "taps_mx.hip", "taps_mx_attend.hip"]


def _commands(out: str) -> list:
    common = [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
              # keep the compiler from forming packed fp32 instructions
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-I", INCLUDE, "-I", CSRC]
    objects = [f"{out}.{s}.o" for s in SOURCES]
    compile_ = [[*common, "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]
    return [*compile_, [*common, "-shared", *objects, "-o", out]]


def build(verbose: bool = False) -> str:
    """Builds libtaps_attention.so (one compiler per source file); returns its path."""
    tmp = LIB + ".tmp"
    *compiles, link = _commands(tmp)
    try:
        running = []
        for cmd in compiles:
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True))
        said = [p.communicate()[0] for p in running]
        if any(p.returncode for p in running):
            sys.stderr.write("".join(said))
            raise RuntimeError(f"building {os.path.basename(LIB)} failed")
        res = subprocess.run(link, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError(f"linking {os.path.basename(LIB)} failed")
        os.replace(tmp, LIB)
    finally:
        for cmd in compiles:
            if os.path.exists(cmd[-1]):
                os.remove(cmd[-1])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
