"""Builds libkvcrush.so (the C-ABI library) from csrc/*.hip for gfx950 with hipcc.

Cross-compiles without a GPU.  The library is written next to this file so that
it travels with the source tree; nothing is installed.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libkvcrush.so")
BENCH_LIB_PATH = os.path.join(PKG_DIR, "libkvcrush_bench.so")   # measurement aids, loaded by bench.py only

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    # packed-fp32 VALU forms are kept out of the generated code on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build_library(verbose: bool = False, extra_flags=()) -> str:
    """The sources are compiled side by side (no kernel of one calls into another) and linked."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]

    def compile_one(source, out):
        cmd = [hipcc, *compile_flags, *extra_flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", "-o", out, source]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        return out

    tmp = LIB_PATH + f".tmp{os.getpid()}"
    with tempfile.TemporaryDirectory() as folder, ThreadPoolExecutor(max(1, min(len(os.sched_getaffinity(0)), 16))) as pool:
        jobs = [pool.submit(compile_one, src, os.path.join(folder, os.path.basename(src) + ".o")) for src in sources()]
        objects = [j.result() for j in jobs]
        subprocess.run([hipcc, *HIPCC_FLAGS, *extra_flags, "-o", tmp, *objects], check=True)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


def build_bench_library() -> str:
    """The benchmark's calibration kernels (csrc/bench/), a library of their own so that the
    product library exports the method's entry points and nothing else."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = BENCH_LIB_PATH + f".tmp{os.getpid()}"
    subprocess.run([hipcc, *HIPCC_FLAGS, "-o", tmp, *sorted(glob.glob(os.path.join(CSRC, "bench", "*.hip")))], check=True)
    os.replace(tmp, BENCH_LIB_PATH)
    return BENCH_LIB_PATH


def ensure_built() -> str:
    """Build the library only if there is none (test harnesses, smoke runs and the benchmark call
    this; the binding itself never builds and raises when the library is missing)."""
    if not os.path.exists(BENCH_LIB_PATH):
        build_bench_library()
    return LIB_PATH if os.path.exists(LIB_PATH) else build_library()


def resource_usage(source: str) -> dict:
    """Compile one csrc file (device code only, no output kept) and return the compiler's
    per-kernel resource report: {mangled kernel name: {"VGPRs": n, "VGPRs Spill": n, ...}}.

    The hand-scheduled score kernels sit close to the register file's limit; a spill there
    costs a multiple of their run time, so the test suite checks this report."""
    import re
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    with tempfile.TemporaryDirectory() as tmp:
        cmd = [hipcc, *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-I",
               os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, source), "-o",
               os.path.join(tmp, "dev.o")]
        out = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    report, cur = {}, None
    for line in out.splitlines():
        m = re.search(r"remark:\s+(.+?):\s+(\S+)\s+\[-Rpass", line)
        if not m:
            continue
        key, val = re.sub(r"\s*\[.*\]$", "", m.group(1).strip()), m.group(2)
        if key == "Function Name":
            cur = report.setdefault(val, {})
        elif cur is not None and val.lstrip("-").isdigit():
            cur[key] = int(val)
    return report


if __name__ == "__main__":
    print(build_library(verbose=True, extra_flags=sys.argv[1:]))
    print(build_bench_library())
