"""Builds liblookahead.so (HIP, gfx950) in-tree with hipcc.

Usage: python -m paper_2602_16760_amd.build [--force]
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "liblookahead.so")

SOURCES = ["la_api.hip", "la_generic.hip", "la_accept.hip", "la_mfma.hip", "la_paged.hip", "la_attend.hip", "la_sample.hip",
           "la_tree.hip", "la_tree_attend.hip", "la_tree_wide.hip", "la_adjust.hip",
           "la_stack_mt1.hip", "la_stack_mt2.hip", "la_stack_mt3.hip", "la_stack_mt4.hip",
           "la_rstack_mt1.hip", "la_rstack_mt2.hip", "la_rstack_mt3.hip", "la_rstack_mt4.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-Wno-unknown-warning-option",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("hipcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = True) -> str:
    """Compiles every source and links liblookahead.so.  LA_EXPERIMENTS=1 in the environment builds
    the variant with device timelines (LA_TRACE) and timing experiments (LA_DBG) compiled in."""
    os.makedirs(OBJ, exist_ok=True)
    flags = FLAGS + (["-DLA_EXPERIMENTS"] if os.environ.get("LA_EXPERIMENTS") == "1" else [])
    stamp = os.path.join(OBJ, "flags.txt")
    if not os.path.exists(stamp) or open(stamp).read() != " ".join(flags):
        force = True  # objects of another variant
        with open(stamp, "w") as fh:
            fh.write(" ".join(flags))
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    headers.append(os.path.join(ROOT, "include", "la.h"))
    hipcc = _hipcc()
    jobs = []
    objs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".hip", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            jobs.append([hipcc, "-x", "hip", "-c", s, "-o", o] + flags)

    def run(cmd):
        if verbose:
            print("[build]", os.path.basename(cmd[4]), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
        bad = [ln for ln in r.stderr.splitlines() if "warning" in ln and "packed-fp32-ops" not in ln]
        if verbose and bad:
            print("\n".join(bad[:20]))

    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(run, jobs))
    if force or jobs or _stale(LIB, objs):
        cmd = [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
        if verbose:
            print("[build] linked", LIB, flush=True)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv)
