"""Build the gfx950 ARC-KV library (libarckv.so) in-tree with hipcc, and the native part of its Python binding
(_arckv_bind.so, host code alone) with the host compiler.

Usage: python -m paper_2609_36835_amd.build  (or build() from Python).
Every call recompiles; objects go to paper_2609_36835_amd/_build/.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libarckv.so")
BIND_SOURCE = os.path.join(PKG, "binding", "bind.cpp")
BIND = os.path.join(PKG, "_arckv_bind.so")
ARCH = "gfx950"

COMMON_FLAGS = [
    "-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
    "-I", INCLUDE, "-I", CSRC,
    # packed fp32 instructions stay off (compiler-generated v_pk_* fp32 ops)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result", "-Wno-unused-command-line-argument",
]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def sources() -> list:
    out = []
    for f in sorted(os.listdir(CSRC)):
        if f.endswith(".hip") or f.endswith(".cpp"):
            out.append(os.path.join(CSRC, f))
    return out


def _compile(src: str, hipcc: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [hipcc, *COMMON_FLAGS, *lang, "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    return obj


def build_binding() -> str:
    """The native part of the Python binding, for the torch that is installed."""
    import torch
    at = os.path.dirname(torch.__file__)
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        raise RuntimeError("no host compiler found")
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(_hipcc())))
    tmp = BIND + ".tmp"
    cmd = [cxx, "-O2", "-fPIC", "-shared", "-std=c++17", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DARCKV_TORCH="{torch.__version__}"', "-I", INCLUDE, "-I", os.path.join(at, "include"),
           "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
           "-I", os.path.join(rocm, "include"), BIND_SOURCE, "-o", tmp, "-L", os.path.join(at, "lib"), "-ltorch_python",
           "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, BIND)
    return BIND


def _binding():
    """build_binding() where a host compiler and torch's headers are at hand.  The library does without: its Python
    binding then goes through ctypes for every call, so none that was built before is left for it to find."""
    try:
        return build_binding()
    except (ImportError, OSError, RuntimeError) as e:
        if os.path.exists(BIND):
            os.remove(BIND)
        print(f"{BIND} not built, calls take some microseconds of host time more: {e}", file=sys.stderr)
        return None


def build(verbose: bool = True, jobs: int = 8) -> str:
    hipcc = _hipcc()
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sources()
    with concurrent.futures.ThreadPoolExecutor(max_workers=max(1, min(jobs, len(srcs) + 1))) as ex:
        binding = ex.submit(_binding)
        objs = list(ex.map(lambda s: _compile(s, hipcc), srcs))
        bound = binding.result()
    tmp = LIB + ".tmp"
    cmd = [hipcc, "-shared", "-fPIC", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources" + (f", and {bound}" if bound else ""), file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
