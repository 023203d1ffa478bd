"""Builds libmixgcn.so (HIP, gfx950) in-tree.  No fallbacks: a missing hipcc is an error."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
BUILD_DIR = os.path.join(_HERE, "_build")
LIB_PATH = os.path.join(_HERE, "libmixgcn.so")

SOURCES = ["abi.hip", "pool.hip", "scan.hip", "sort.hip", "csr.hip", "spmm.hip", "rowgroups.hip", "gemm.hip", "gemm_rows.hip", "gemm_rows_f32.hip",
           "gemm_bf16.hip", "gemm_bf16_deep.hip", "gemm_split.hip", "gemm_split_forward.hip", "loss.hip", "linear_xent.hip",
           "checkpoint.hip", "peaks.hip",
           "reorder.hip"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    # packed fp32 VALU ops are kept off on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(_ROOT, "include"), "-I", CSRC,
]


def _hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return exe


def _newer(src: str, out: str) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    deps = [src] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    deps.append(os.path.join(_ROOT, "include", "mixgcn.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, extra_flags=(), out: str = LIB_PATH,
          build_dir: str = BUILD_DIR) -> str:
    """extra_flags / out / build_dir let an experiment build a variant next to the product."""
    os.makedirs(build_dir, exist_ok=True)
    hipcc = _hipcc()
    objs = []
    jobs = []
    for name in SOURCES:
        src = os.path.join(CSRC, name)
        obj = os.path.join(build_dir, name.replace(".hip", ".o"))
        objs.append(obj)
        if force or _newer(src, obj):
            jobs.append([hipcc, *HIPCC_FLAGS, *extra_flags, "-c", src, "-o", obj])

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
        warn = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l and l.strip())
        if verbose and warn:
            print(warn, flush=True)

    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        list(ex.map(run, jobs))
    if jobs or not os.path.exists(out):
        run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", out, *objs])
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
