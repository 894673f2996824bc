"""Build libtc_mi355x.so (hipcc, gfx950 only) next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtc_mi355x.so")
SCHED_LIB = os.path.join(HERE, "libtc_sched.so")  # host-only scheduling core, built with the host compiler
SOURCES = ["tc_plan.cpp", "tc_api.cpp", "tc_kernels.hip", "tc_kvq.hip", "tc_rows.hip", "tc_span.hip", "tc_span_plan.cpp", "tc_probe.hip"]
LINK_FLAGS = ["--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-command-line-argument"]


TRACE_LIB = os.path.join(HERE, "libtc_mi355x_trace.so")  # the same library with per-workgroup time stamps in the attention kernel


def build(verbose: bool = False, extra=(), trace: bool = False) -> str:
    """Every source into an object of its own, side by side (the two files of kernels take most of the time), then one library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if trace:
        extra = [*extra, "-DTC_WG_TRACE"]
    lib = TRACE_LIB if trace else LIB
    noise = "is not a recognized feature for this target"

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + err)
        if verbose and err.strip():
            print(err)

    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_one = [[hipcc, *FLAGS, *extra, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", "-x", "hip", os.path.join(CSRC, s), "-o", o]
                       for s, o in zip(SOURCES, objects)]
        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as pool:
            list(pool.map(run, compile_one))
        run([hipcc, *LINK_FLAGS, *objects, "-o", lib])
    return lib


def build_sched(verbose: bool = False) -> str:
    """The scheduling core has no GPU code: plain g++, so it also loads where no ROCm runtime is."""
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wextra", "-ffp-contract=off",
           "-I", os.path.join(ROOT, "include"), os.path.join(CSRC, "tc_sched.cpp"), "-o", SCHED_LIB]
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed:\n" + r.stderr)
    if verbose and r.stderr.strip():
        print(r.stderr)
    return SCHED_LIB


if __name__ == "__main__":
    print(build_sched(verbose=True))
    if "--trace" in sys.argv[1:]:
        print(build(verbose=True, trace=True))
    else:
        print(build(verbose=True, extra=[a for a in sys.argv[1:] if a.startswith("-")]))
