"""Build libnsgcqt.so in-tree for gfx950.

The host plan builder is plain C++ (g++); the kernels and the C ABI are HIP
(hipcc). Every HIP translation unit is compiled with packed-FP32 instructions
disabled. Usage: ``python -m paper_2609_29119_amd.build`` or ``build()``.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libnsgcqt.so")
ARCH = os.environ.get("NSGCQT_ARCH", "gfx950")

HIP_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-Wno-gnu-zero-variadic-macro-arguments",
]

# The layers are compiled at -O2: at -O3 one instantiation of the 32-bit
# per-band product is unrolled until it spills (3.5 KB a lane).
LAYER_FLAGS = [f if f != "-O3" else "-O2" for f in HIP_FLAGS]
LAYERS = ["linear", "rotary", "attention", "attention_grad", "step", "decay", "norm", "gated"]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"build step failed: {' '.join(cmd[:3])} ...")
    return r


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library; returns its path."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    os.makedirs(BUILD, exist_ok=True)
    _run([sys.executable, os.path.join(CSRC, "gen_radix_consts.py"), os.path.join(CSRC, "radix_consts.hpp")],
         verbose)
    plan_o = os.path.join(BUILD, "plan.o")
    hip_o = os.path.join(BUILD, "nsgcqt.o")
    jobs = [["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-c", os.path.join(CSRC, "plan.cpp"), "-o", plan_o],
            [hipcc, *HIP_FLAGS, "-c", os.path.join(CSRC, "nsgcqt.hip"), "-o", hip_o]]
    objects = [plan_o, hip_o]
    for name in LAYERS:
        objects.append(os.path.join(BUILD, f"layers_{name}.o"))
        jobs.append([hipcc, *LAYER_FLAGS, "-c", os.path.join(CSRC, "layers", f"{name}.hip"), "-o", objects[-1]])
    with ThreadPoolExecutor(min(len(jobs), os.cpu_count() or 1)) as pool:
        list(pool.map(lambda cmd: _run(cmd, verbose), jobs))
    tmp = LIB + ".tmp"
    _run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objects], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
