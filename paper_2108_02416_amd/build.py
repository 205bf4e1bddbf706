"""Build libaspis.so (gfx950) in-tree with hipcc, and the binding's Python
module _tensors.so with g++.

The library is the C ABI declared in include/aspis.h: host code
(csrc/aspis_host.cpp, csrc/aspis_sim.cpp) plus the HIP kernels
(csrc/aspis_kernels.hip, and csrc/aspis_ws_*.hip for the warp-specialised
kernels' many instantiations).  _tensors (csrc/aspis_tensors.cpp) reads the
addresses and layouts of torch tensors.
"""
import importlib.util
import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libaspis.so")
TENSORS = os.path.join(HERE, "_tensors.so")
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
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed building {cmd[cmd.index('-o') + 1]}")
    return msgs


def _tensors_command() -> list[str]:
    # found without importing torch: its path is all that is needed
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wno-unused-function",
            "-I", os.path.join(torch, "include"),
            "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
            "-I", sysconfig.get_paths()["include"],
            "-o", TENSORS + ".tmp", os.path.join(HERE, "csrc", "aspis_tensors.cpp"),
            "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def build(verbose: bool = False) -> str:
    """Compile the sources in parallel (one object each) and link them."""
    flags = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall",
             "-Wno-unused-function", "-I", os.path.join(ROOT, "include"), *DEVICE_FLAGS]
    with tempfile.TemporaryDirectory() as tmp:
        cmds, objs = [], []
        for src in SOURCES:
            objs.append(os.path.join(tmp, src + ".o"))
            cmds.append([HIPCC, *flags, "-c", "-o", objs[-1], os.path.join(HERE, "csrc", src)])
        cmds.append(_tensors_command())
        link = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB + ".tmp", *objs]
        if verbose:
            print("\n".join(" ".join(c) for c in [*cmds, link]), flush=True)
        with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:
            msgs = [m for ms in pool.map(_run, cmds) for m in ms]
        msgs += _run(link)
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(LIB + ".tmp", LIB)
    os.replace(TENSORS + ".tmp", TENSORS)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
