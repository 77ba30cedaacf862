"""Compile the HIP sources of the rTop-k library into ``librtopk.so`` (gfx950)."""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "librtopk.so")
# the same sources with RTOPK_DEBUG_CHECKS: the master entry points verify their
# preconditions (index range, ascending slices) on the device before they launch
DEBUG_LIB_PATH = os.path.join(HERE, "librtopk_debug.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950",
    # packed-fp32 instruction selection is kept off for every device function
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fPIC", "-shared",
]


def sources() -> list:
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _run(cmd: list, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # hipcc's host pass warns that it does not know the device-only target feature
    noise = ("packed-fp32-ops", "is not a recognized feature")
    out = "\n".join(l for l in res.stdout.splitlines() if not any(n in l for n in noise))
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out, flush=True)


def build(verbose: bool = False, debug: bool = False) -> str:
    """Compiles every source, several at once, and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out_path = DEBUG_LIB_PATH if debug else LIB_PATH
    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"] + (["-DRTOPK_DEBUG_CHECKS"] if debug else [])
    with tempfile.TemporaryDirectory() as folder:
        jobs = [(src, os.path.join(folder, os.path.basename(src) + ".o")) for src in sources()]
        with concurrent.futures.ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 1, 8)) as pool:
            list(pool.map(lambda job: _run([hipcc] + compile_flags + ["-c", "-o", job[1], job[0]], verbose), jobs))
        _run([hipcc] + HIPCC_FLAGS + ["-o", out_path] + [obj for _, obj in jobs], verbose)
    return out_path


if __name__ == "__main__":
    print(build(verbose="-q" not in sys.argv, debug="--debug" in sys.argv))
