"""Build libnnconv.so (HIP, gfx950) in-tree with hipcc.

    python -m paper_2102_06725_amd.build

Compiles every ``csrc/*.hip`` file to an object under ``_build/`` in
parallel and links them into ``paper_2102_06725_amd/libnnconv.so``.

``libnnconv_recompute.so`` is the same library for tests, with recurrence
kernels whose workgroups do not wait for each other's words and compute all
of them again instead: the path that a wait takes when it gives up.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libnnconv.so")
RECOMPUTE_LIB = os.path.join(PKG, "libnnconv_recompute.so")
RECOMPUTE = {"recurrence_fwd.hip": ["-DNNCONV_RECURRENCE_LOOKS=0"], "recurrence_bwd.hip": ["-DNNCONV_RECURRENCE_LOOKS=0"]}
ARCH = "gfx950"

CXXFLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    "--offload-arch=" + ARCH,
    # keep the compiler from emitting packed fp32 math
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libnnconv)")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def link(objs, lib) -> None:
    tmp = lib + ".tmp%d" % os.getpid()
    subprocess.run([hipcc(), "--offload-arch=" + ARCH, "-shared", "-fPIC", "-o", tmp] + objs, check=True)
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    """Compile and link; always rebuilds.  Returns the library path."""
    cc = hipcc()
    os.makedirs(BUILD, exist_ok=True)
    procs = []
    objs, again = [], []

    def compile_to(src, name, flags):
        obj = os.path.join(BUILD, name + ".o")
        cmd = [cc] + CXXFLAGS + flags + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        return obj

    for src in sources():
        base = os.path.basename(src)
        objs.append(compile_to(src, base[:-4], []))
        again.append(compile_to(src, base[:-4] + "_recompute", RECOMPUTE[base]) if base in RECOMPUTE else objs[-1])
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = "\n".join(l for l in out.decode(errors="replace").splitlines()
                         if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            failed.append((src, text))
        elif verbose and text.strip():
            print(text)
    if failed:
        msg = "\n".join("%s:\n%s" % (s, t) for s, t in failed)
        raise RuntimeError("libnnconv build failed:\n" + msg)
    link(objs, LIB)
    link(again, RECOMPUTE_LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
