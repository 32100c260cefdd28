"""Compile ``csrc/`` into ``libcorun.so`` for gfx950 with hipcc, in-tree.

Run as ``python -m paper_2608_14376_amd.build``.  It always recompiles.
"""
from __future__ import annotations

import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcorun.so")
SOURCES = ["kernels.hip", "cache.hip", "beam.hip", "pages.hip", "shared.hip", "engine.cpp", "cache_ops.cpp",
           "group_ops.cpp", "scheduler.cpp", "sample_noalloc.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-fp32 instructions are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def scratch_of(remarks: str) -> dict:
    """{kernel: bytes of scratch per lane}, of those that have any, from the
    compiler's kernel-resource-usage remarks."""
    found, name = {}, ""
    for ln in remarks.splitlines():
        m = re.search(r"remark:\s+(Function Name|ScratchSize \[bytes/lane\]): (\S+)", ln)
        if m and m[1] == "Function Name":
            name = m[2]
        elif m and m[2] != "0":
            found[name] = int(m[2])
    return found


def compile_object(src: str, obj: str, verbose: bool = False) -> None:
    """One source to an object file.  A kernel with scratch memory is refused:
    kernels that load straight into LDS have faulted with spilled registers,
    and none of the others needs any."""
    cmd = [HIPCC, *FLAGS, "-Rpass-analysis=kernel-resource-usage", "-c", "-x", "hip", src,
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    lines = (r.stdout + r.stderr).splitlines()
    # a remark is followed by its source line and a mark under it
    noise = {i + j for i, ln in enumerate(lines) if "[-Rpass-analysis=kernel-resource-usage]" in ln for j in range(3)
             if j == 0 or re.match(r"\s*\d*\s*\|", lines[i + j] if i + j < len(lines) else "")}
    msgs = [ln for i, ln in enumerate(lines) if i not in noise and "packed-fp32-ops' is not a recognized feature" not in ln]
    if msgs and (verbose or r.returncode):
        print("\n".join(msgs), file=sys.stderr)
    if r.returncode:
        raise RuntimeError(f"hipcc failed on {os.path.basename(src)}")
    scratch = scratch_of(r.stdout + r.stderr)
    if scratch:
        raise RuntimeError(f"{os.path.basename(src)}: kernels with scratch memory: {scratch}")


def build(verbose: bool = False) -> str:
    objs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        compile_object(os.path.join(CSRC, src), obj, verbose)
        objs.append(obj)
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    for o in objs:
        os.remove(o)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
