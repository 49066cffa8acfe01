"""Build libsparseinfer.so (HIP, gfx950) and _autograd.so (host code) in-tree.

Usage: ``python -m paper_2411_12692_amd.build`` (or ``__graft_entry__.build()``).
``python -m paper_2411_12692_amd.build --trace`` builds the phase-trace
variant ``libsparseinfer_trace.so`` instead (the row-owning kernel compiled
with ``-DSI_TRACE``, read by ``paper_2411_12692_amd.phase_trace``).
"""

from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libsparseinfer.so")
TRACE_LIB = os.path.join(PKG, "libsparseinfer_trace.so")
AUTOGRAD_LIB = os.path.join(PKG, "_autograd.so")
TRACED = "owned.hip"  # the source compiled with -DSI_TRACE in the trace variant
SOURCES = ["api.hip", "pack.hip", "predict.hip", "mlp.hip", "owned.hip", "diag.hip",
           "mx_quant.hip", "mx_linear.hip", "mx_sparse.hip", "mx_api.hip", "norm.hip",
           "dense.hip", "dense_rr.hip", "dense_gated.hip", "dense_cr.hip", "dense_dh.hip", "dense_cc.hip", "dense_fp8.hip",
           "dense_few.hip", "fp8.hip", "norm_train.hip", "dense_api.hip"]
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else "hipcc")

CXX = os.environ.get("CXX", "g++")

# Packed-FP32 instructions are disabled: compile plain scalar float code only.
COMMON = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics",
    "-I", os.path.join(ROOT, "include"),
]


def _run(cmd):
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in p.stdout.splitlines() if "packed-fp32-ops" not in l)
    if p.returncode != 0:
        raise RuntimeError(f"command failed ({p.returncode}): {' '.join(cmd)}\n{out}")
    return out


def autograd_lacks() -> str:
    """What building the nodes of PyTorch's graph asks for beyond hipcc and is not here
    ("" where nothing is missing)."""
    if shutil.which(CXX) is None:
        return f"a C++ compiler ({CXX})"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python's headers"
    from torch.utils.cpp_extension import include_paths
    if not any(os.path.exists(os.path.join(p, "torch", "csrc", "autograd", "function.h")) for p in include_paths()):
        return "PyTorch's headers"
    return ""


def build_autograd() -> str:
    """Compile and link the nodes of PyTorch's graph (``csrc/autograd.cpp``, host code
    beside the library, which it finds in its own folder)."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    os.makedirs(BUILD, exist_ok=True)
    obj = os.path.join(BUILD, "autograd.o")
    include = [f"-I{p}" for p in (*include_paths(), sysconfig.get_paths()["include"])]
    _run([CXX, "-O2", "-std=c++17", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          *include, "-c", os.path.join(CSRC, "autograd.cpp"), "-o", obj])
    tmp = AUTOGRAD_LIB + ".tmp"
    _run([CXX, "-shared", obj, "-o", tmp, f"-L{PKG}", "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN",
          *[f"-L{p}" for p in library_paths()], "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python"])
    shutil.move(tmp, AUTOGRAD_LIB)
    return AUTOGRAD_LIB


def build(verbose: bool = False, trace: bool = False) -> str:
    """Compile every HIP source and link the shared library (``trace``: the
    phase-trace variant), then the nodes of PyTorch's graph; returns the library's
    path.  The library asks for hipcc alone: where the nodes cannot be built it is
    complete without them (the C ABI, and every call without gradients), which is said
    on stderr, and calls that need them raise."""
    out_dir = os.path.join(BUILD, "trace") if trace else BUILD
    lib = TRACE_LIB if trace else LIB
    os.makedirs(out_dir, exist_ok=True)
    objs = []
    jobs = []
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        for src in SOURCES:
            obj = os.path.join(out_dir, os.path.splitext(src)[0] + ".o")
            objs.append(obj)
            extra = ["-DSI_TRACE"] if trace and src == TRACED else []
            cmd = [HIPCC, *COMMON, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
            jobs.append(ex.submit(_run, cmd))
        for j in jobs:
            out = j.result()
            if verbose and out.strip():
                print(out)
    tmp = lib + ".tmp"
    _run([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp])
    shutil.move(tmp, lib)
    if not trace:
        lacks = autograd_lacks()
        if lacks:
            if os.path.exists(AUTOGRAD_LIB):  # of other sources
                os.remove(AUTOGRAD_LIB)
            print(f"{os.path.basename(AUTOGRAD_LIB)} is not built, gradients are not available: {lacks} missing",
                  file=sys.stderr)
        else:
            build_autograd()
    return lib


if __name__ == "__main__":
    path = build(verbose=True, trace="--trace" in sys.argv[1:])
    print(path)
    sys.exit(0)
