"""Compile the HIP sources under ``csrc/`` into ``libhd.so`` for gfx950.

Each translation unit is compiled on its own (in parallel), then linked into
one shared library with a plain C ABI (``include/hd.h``).
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import re
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libhd.so")
ARCH = os.environ.get("HD_OFFLOAD_ARCH", "gfx950")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CFLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # Packed fp32 VALU instructions stay off: hipcc would otherwise form them
    # from ordinary float code.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result", "-Wno-unknown-pragmas",
    "-I", os.path.join(ROOT, "include"),
]


# Kernels under csrc/ops keep their accumulators and loads in flight in registers. Instances that
# did not fit (scratch memory in use) have given wrong sums with this compiler, without
# an error, so a build in which one appears is refused.
OPS = os.path.join(CSRC, "ops")
RESOURCES = "-Rpass-analysis=kernel-resource-usage"


def spilling(remarks: str) -> list:
    """The kernels that use scratch memory, from the compiler's resource remarks."""
    names, name = [], "?"
    for line in remarks.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
        m = re.search(r"ScratchSize \[bytes/lane\]: (\d+)|Dynamic Stack: (True)", line)
        if m and m.group(1) != "0":
            names.append(name)
    return names


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    in_registers = os.path.dirname(os.path.abspath(src)) == OPS
    cmd = [HIPCC, *CFLAGS, *([RESOURCES] if in_registers else []), "-c", src, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and "not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{out}")
    if in_registers:
        spilled = spilling(out)
        if spilled:
            os.remove(obj)
            raise RuntimeError(f"{src}: kernels that do not fit their registers: {spilled}")
        out = "\n".join(l for l in out.splitlines() if "warning:" in l)  # (not the remarks)
    if verbose and out.strip():
        print(out, flush=True)
    return obj


def build(verbose: bool = False, jobs: int = 0) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip"))
                  + glob.glob(os.path.join(CSRC, "ops", "*.hip")))
    jobs = jobs or min(8, os.cpu_count() or 4)
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


FLOORS_SRC = os.path.join(ROOT, "bench_floors.hip")
FLOORS_LIB = os.path.join(ROOT, "bench_floors.so")


def build_floors(verbose: bool = False) -> str:
    """The benchmark's measurement-floor kernels (bench_floors.hip, beside
    bench.py): not part of libhd.so."""
    tmp = FLOORS_LIB + ".tmp"
    cmd = [HIPCC, *CFLAGS, "-shared", FLOORS_SRC, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {FLOORS_SRC}:\n{r.stdout}{r.stderr}")
    os.replace(tmp, FLOORS_LIB)
    return FLOORS_LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
