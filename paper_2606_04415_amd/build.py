"""Build libflexattn.so (HIP kernels + C ABI) for gfx950 in-tree.

``python -m paper_2606_04415_amd.build`` compiles every source with hipcc into
``paper_2606_04415_amd/libflexattn.so``. Objects are built in parallel and
linked into one shared library; the planner (plan.cpp) is plain host C++ in
the same library.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libflexattn.so")
SOURCES = ["attention.hip", "decode_kv8.hip", "prefill_kv8.hip", "latent.hip", "kv_append.hip", "api.hip", "plan.cpp", "controller.cpp"]
# sources whose values may be NaN: what they copy or quantise is the caller's
KEEPS_NANS = {"kv_append.hip"}
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libflexattn.so)")


def common_flags(src: str = ""):
    flags = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
             # keep the compiler from forming packed fp32 VALU instructions
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-function"]
    if src not in KEEPS_NANS:
        # scores are finite; max() needs no NaN quieting (a NaN from a wrong
        # page still reaches the output through the P x V product)
        flags.append("-fno-honor-nans")
    return flags


def build(verbose: bool = False) -> str:
    cc = hipcc()
    bdir = os.path.join(PKG, "_build")
    os.makedirs(bdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(bdir, os.path.splitext(src)[0] + ".o")
        cmd = [cc] + common_flags(src) + ["-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cpp"):
            cmd = [cc, "-x", "hip"] + cmd[1:]
        r = subprocess.run(cmd, capture_output=True, text=True)
        msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                         if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{msgs}")
        if verbose and msgs.strip():
            print(msgs, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
