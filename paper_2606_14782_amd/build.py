"""Builds libbacon.so (the gfx950 kernels and the C ABI) in-tree with hipcc."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbacon.so")
SOURCES = ["kernels.hip", "noalloc.hip", "cache.hip", "cache4.hip", "cache_attend.hip", "prompt.hip", "rotary.hip",
           "api.cpp", "cache_api.cpp", "prompt_api.cpp", "rotary_api.cpp"]

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU forms are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # inputs are finite (the method has no NaN semantics); this lets the
    # max of logits skip the NaN-quieting operand copies
    "-fno-honor-nans",
    "-Wall", "-Wno-unused-result",
]
# attention hands a NaN on to the outputs of its query, a rotation passes one as it is
# (and its host side refuses NaN in its numbers)
SOURCE_FLAGS = {s: ["-fhonor-nans"] for s in ("cache_attend.hip", "prompt.hip", "rotary.hip", "rotary_api.cpp")}


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False) -> str:
    """Compile every source into ``paper_2606_14782_amd/libbacon.so`` (always rebuilds)."""
    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
        if verbose:
            print(" ".join(cmd))

    cc, include, tmp = hipcc(), os.path.join(HERE, "..", "include"), LIB + ".tmp"
    with tempfile.TemporaryDirectory() as objs, concurrent.futures.ThreadPoolExecutor(4) as pool:
        out = {s: os.path.join(objs, s + ".o") for s in SOURCES}
        jobs = [[cc, *HIP_FLAGS, *SOURCE_FLAGS.get(s, []), "-I", include, "-c", os.path.join(CSRC, s), "-o", out[s]]
                for s in SOURCES]
        list(pool.map(run, jobs))
        run([cc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *out.values()])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
