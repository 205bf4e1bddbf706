"""Build libaspis.so (gfx950) in-tree with hipcc.

The library is the C ABI declared in include/aspis.h: host code
(csrc/aspis_host.cpp, csrc/aspis_sim.cpp) plus the HIP kernels
(csrc/aspis_kernels.hip, and csrc/aspis_ws_*.hip for the warp-specialised
kernels' many instantiations).
"""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libaspis.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

# Packed-fp32 instructions are disabled for all device code (the kernels
# here are integer and fp64 work; this keeps the compiler from forming
# v_pk_* fp32 forms from any float code).
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


SOURCES = ["aspis_host.cpp", "aspis_sim.cpp", "aspis_clip.cpp", "aspis_clip.hip",
           "aspis_kernels.hip", "aspis_ws_r3.hip", "aspis_ws_r3_table.hip", "aspis_ws_r5.hip",
           "aspis_ws_r7.hip", "aspis_ws_median.hip"]


def _run(cmd: list[str]) -> list[str]:
    """Run one compiler command; returns its messages, raises on failure."""
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the device feature named in DEVICE_FLAGS
    msgs = [ln for ln in (r.stdout + r.stderr).splitlines()
            if "packed-fp32-ops" not in ln and ln.strip()]
    if r.returncode != 0:
        sys.stderr.write("\n".join(msgs) + "\n")
        raise RuntimeError("hipcc failed building libaspis.so")
    return msgs


def build(verbose: bool = False) -> str:
    """Compile the sources in parallel (one object each) and link them."""
    flags = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall",
             "-Wno-unused-function", "-I", os.path.join(ROOT, "include"), *DEVICE_FLAGS]
    with tempfile.TemporaryDirectory() as tmp:
        cmds, objs = [], []
        for src in SOURCES:
            objs.append(os.path.join(tmp, src + ".o"))
            cmds.append([HIPCC, *flags, "-c", "-o", objs[-1], os.path.join(HERE, "csrc", src)])
        link = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB + ".tmp", *objs]
        if verbose:
            print("\n".join(" ".join(c) for c in [*cmds, link]), flush=True)
        with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:
            msgs = [m for ms in pool.map(_run, cmds) for m in ms]
        msgs += _run(link)
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
