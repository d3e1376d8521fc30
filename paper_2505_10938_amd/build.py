"""Build the C-ABI library (libkvq.so) in-tree with hipcc for gfx950."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libkvq.so")

SOURCES = ["kvq_api.hip", "kvq_quantize.hip", "kvq_trace.hip", "kvq_decode.hip", "kvq_dequant.hip",
           "kvq_prompt.hip", "kvq_extend.hip", "kvq_pages.hip", "kvq_rope.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + proc.stdout + proc.stderr)
    if verbose and proc.stderr:
        print(proc.stderr)


def build_library(verbose: bool = False) -> str:
    """Compile every HIP source into paper_2505_10938_amd/libkvq.so and return its path.  The sources are compiled
    side by side (a build takes as long as the decode kernel's, not as all of them), then linked."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as work, concurrent.futures.ThreadPoolExecutor(4) as pool:
        objects = [os.path.join(work, s.replace(".hip", ".o")) for s in SOURCES]
        jobs = [pool.submit(_run, [hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                                   os.path.join(CSRC, s), "-o", o], verbose) for s, o in zip(SOURCES, objects)]
        for job in jobs:
            job.result()
        _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB_PATH], verbose)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
