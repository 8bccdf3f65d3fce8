"""Build the HIP library libbirkhoff4.so for gfx950, in-tree (no JIT cache).

Usage: python -m paper_2606_07574_amd.build   (or call build()).
"""
from __future__ import annotations

import os
import shutil
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SOURCES = [os.path.join(PKG, "csrc", f) for f in ("birkhoff4.hip", "pre.hip")]
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libbirkhoff4.so")
ARCH = "gfx950"

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # keep packed-fp32 instructions out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # fp32 denormals flush to zero (the forward kernel relies on it, see csrc)
    "-fgpu-flush-denormals-to-zero",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return path


def build(extra_flags: list[str] | None = None, out: str = LIB, verbose: bool = False) -> str:
    """Compile the sources in csrc/ and link them into ``out`` (always recompiles)."""
    objs = [out + ".%s.tmp%d.o" % (os.path.basename(s), os.getpid()) for s in SOURCES]
    tmp = out + ".tmp%d" % os.getpid()
    cmds = [[hipcc(), *FLAGS, *(extra_flags or []), "-I", INCLUDE, "-c", "-o", o, s] for s, o in zip(SOURCES, objs)]
    link = [hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs]
    if verbose:
        print("\n".join(" ".join(c) for c in (*cmds, link)), flush=True)
    try:
        jobs = [subprocess.Popen(c) for c in cmds]
        codes = [j.wait() for j in jobs]  # every compiler has ended before any error is raised
        for c, code in zip(cmds, codes):
            if code:
                raise subprocess.CalledProcessError(code, c)
        subprocess.check_call(link)
        os.replace(tmp, out)
    finally:
        for f in (*objs, tmp):
            if os.path.exists(f):
                os.remove(f)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
