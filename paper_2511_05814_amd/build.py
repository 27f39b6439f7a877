"""Build the HIP library in-tree: paper_2511_05814_amd/_lib/libmoe_offload.so.

Compiles every HIP source under csrc/ for gfx950 with hipcc into one shared
library exporting the C ABI of include/moe_offload.h, and csrc/attention_ops.cpp
(host code: the torch calls of `attention`) into a CPython module beside it that
links to it (with torch only: the C library builds without).  Run as a module
(`python -m paper_2511_05814_amd.build`) or through __graft_entry__.build().
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_lib")
OUT = os.path.join(OUT_DIR, "libmoe_offload.so")
OPS = os.path.join(OUT_DIR, "_attention_ops.so")
ARCH = "gfx950"

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", f"--offload-arch={ARCH}",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def build_ops(verbose: bool = False) -> Optional[str]:
    """The CPython module, against this interpreter's and torch's headers; None
    without torch, for which it is: the C library needs none."""
    import sysconfig

    try:
        import torch
        from torch.utils import cpp_extension
    except ImportError:
        print("torch is not installed: the C library is built without the module of torch calls", file=sys.stderr)
        return None
    tmp = OPS + ".tmp"
    cmd = [hipcc(), "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
           *[f for d in cpp_extension.include_paths() for f in ("-isystem", d)],
           os.path.join(CSRC, "attention_ops.cpp"), "-x", "none", "-o", tmp, OUT, "-Wl,-rpath,$ORIGIN",
           *["-L" + d for d in cpp_extension.library_paths()], "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(res.stderr.splitlines()[-60:]))
    os.replace(tmp, OPS)
    return OPS


def build(verbose: bool = False) -> str:
    os.makedirs(OUT_DIR, exist_ok=True)
    sources = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    tmp = OUT + ".tmp"
    # MOE_HIPCC_EXTRA: extra compiler flags for tuning builds (e.g. -DMOE_FETCH_BLOCKS=32)
    extra = os.environ.get("MOE_HIPCC_EXTRA", "").split()
    # a name of its own, so that what links to it finds the library beside itself, wherever that is
    name = "-Wl,-soname," + os.path.basename(OUT)
    cmd = [hipcc(), *FLAGS, name, *extra, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sources, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    errs = [l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(errs[-60:]))
    if verbose and errs:
        print("\n".join(errs[-40:]))
    os.replace(tmp, OUT)
    build_ops(verbose)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
