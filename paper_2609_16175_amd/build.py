"""Build step of libboa.so (hipcc, gfx950). Run by __graft_entry__.build()."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SOURCES = [os.path.join(PKG, "csrc", f) for f in ("boa_kernels.hip", "boa_build.hip", "boa_api.hip",
                                                   "boa_norm.hip", "boa_xent.hip", "boa_matvec.hip",
                                                   "boa_linear.hip", "boa_block.hip", "boa_orth.hip")]
LIB = os.path.join(PKG, "libboa.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # distances rely on explicit fused multiply-adds and nothing else fused
    "-ffp-contract=off",
    # no packed-FP32 instructions in generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(PKG, "csrc"),
]


def build(verbose: bool = False, stage_profile: bool = False) -> str:
    """Compile libboa.so; stage_profile=True builds libboa_stageprof.so, a
    variant that prints per-stage cycle counts of every phase to stderr."""
    lib = LIB if not stage_profile else os.path.join(PKG, "libboa_stageprof.so")
    tmp = lib + f".tmp{os.getpid()}"
    flags = [*HIPCC_FLAGS, *(["-DBOA_STAGE_PROFILE"] if stage_profile else [])]

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + r.stdout + r.stderr)
        return r.stderr

    with tempfile.TemporaryDirectory() as d, ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(d, os.path.basename(s) + ".o") for s in SOURCES]
        said = list(pool.map(lambda s, o: run(["hipcc", *flags, "-c", s, "-o", o]), SOURCES, objects))
        said.append(run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", tmp]))
    if verbose:
        print("".join(said))
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose=True))
