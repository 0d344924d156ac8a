"""Builds libmuon_hip.so (the C-ABI library) for gfx950 with hipcc, in-tree.

    python -m paper_2609_21594_amd.csrc.build [--verbose]

Packed fp32 instructions are disabled for all device code (the compiler would
otherwise form v_pk_* fp32 ops from ordinary float code).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(HERE)
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libmuon_hip.so")
SOURCES = ["muon_api.hip", "muon_kernels.hip", "attention_api.hip", "attention_kernels.hip"]
ARCH = os.environ.get("MUON_HIP_ARCH", "gfx950")


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def commands(out: str, objects: str):
    """One command for each source, and the one that links their objects."""
    flags = [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include")]
    objs = [os.path.join(objects, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    return ([[*flags, "-c", os.path.join(HERE, s), "-o", o] for s, o in zip(SOURCES, objs)],
            [hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", *objs, "-o", out])


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    noise = "is not a recognized feature for this target"

    def finish(cmd, run):
        _, err = run.communicate()
        err = "\n".join(l for l in err.splitlines() if noise not in l)
        if run.returncode != 0:
            raise RuntimeError(f"hipcc failed ({run.returncode}): {' '.join(cmd)}\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    def start(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True)

    with tempfile.TemporaryDirectory() as objects:
        compiles, link = commands(tmp, objects)
        runs = [start(c) for c in compiles]  # at once: the kernels take minutes one after the other
        try:
            for c, r in zip(compiles, runs):
                finish(c, r)
        finally:
            for r in runs:
                if r.poll() is None:
                    r.kill()
                    r.wait()
        finish(link, start(link))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="--verbose" in sys.argv))
