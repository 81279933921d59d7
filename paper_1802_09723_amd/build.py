"""Build the HIP library (gfx950) in-tree: paper_1802_09723_amd/lib/librrm_hip.so."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIBDIR, "librrm_hip.so")
SOURCES = ["rrm_api.hip", "scan.hip", "conv_gather.hip", "conv_pos.hip", "conv_scatter.hip", "fc.hip", "fc_batched.hip", "bin_conv.hip", "aux.hip", "probe.hip",
           "group_norm.hip", "gated_scan.hip", "gated_ff.hip", "rrm_ops.hip"]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC", "-shared", "-fvisibility=hidden",
    "-munsafe-fp-atomics",
    # no wave-level aggregation of atomics: it reads the result back at once (a wait for the memory round
    # trip), while the kernels issue their few atomics from one lane and need the result late or never
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build_lib(verbose: bool = False) -> str:
    """A source file a compiler, as many at once as MAX_JOBS (or the CPUs) allow, then one link."""
    os.makedirs(LIBDIR, exist_ok=True)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    jobs = max(1, min(len(SOURCES), int(os.environ.get("MAX_JOBS", "0") or 0) or len(os.sched_getaffinity(0))))

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory(prefix="rrm_build_") as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_flags = [f for f in FLAGS if f != "-shared"] + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        with ThreadPoolExecutor(jobs) as pool:
            list(pool.map(lambda so: run([hipcc] + compile_flags + ["-c", os.path.join(CSRC, so[0]), "-o", so[1]]), zip(SOURCES, objects)))
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", LIB])
    return LIB


if __name__ == "__main__":
    print(build_lib(verbose="-v" in sys.argv))
