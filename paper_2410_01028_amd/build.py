"""Compile the HIP engine for gfx950 into paper_2410_01028_amd/libasd.so (in-tree)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", n) for n in ("asd_engine.hip", "asd_kv.hip", "asd_kv_spans.hip")]
LIB = os.path.join(HERE, "libasd.so")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU forms are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result", "-Wno-unused-value",
    # leading scalar kernel arguments arrive in SGPRs with the wave instead of through a load from the argument segment
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
]


def build(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SRCS]
        cmds = [["hipcc", *FLAGS, "-c", src, "-o", obj] for src, obj in zip(SRCS, objs)]
        _run(cmds, verbose)                                    # the sources side by side
        _run([["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]], verbose)
    return LIB


def _run(cmds: list, verbose: bool) -> None:
    noise = "is not a recognized feature for this target"
    if verbose:
        for cmd in cmds:
            print(" ".join(cmd), flush=True)
    procs = [subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True) for cmd in cmds]
    errs = ["\n".join(l for l in p.communicate()[1].splitlines() if noise not in l) for p in procs]
    if any(p.returncode for p in procs):
        sys.stderr.write("\n".join(errs) + "\n")
        raise RuntimeError("hipcc failed")
    if verbose and any(e.strip() for e in errs):
        print("\n".join(errs))


if __name__ == "__main__":
    print(build(verbose=True))
