"""Build libsfa.so (HIP, gfx950) in-tree.

    python -m paper_2603_22300_amd.build

Compiles every source under csrc/ with hipcc for gfx950 and links the shared
library next to this file; then the native marshalling of the newer entry points,
_binding.so (host code only, against torch's headers).  Always rebuilds (a few seconds
per file)."""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsfa.so")
BINDING = os.path.join(HERE, "_binding.so")
SOURCES = ["sfa_encode.hip", "sfa_fwd.hip", "sfa_fwd_generic.hip", "sfa_fwd_index.hip", "sfa_bwd.hip", "sfa_bwd_generic.hip", "sfa_decode.hip",
           "sfa_decode_generic.hip", "sfa_decode_q8.hip", "sfa_decode_q4.hip",
           "sfa_cache.hip", "sfa_cache_q4.hip", "sfa_pages.hip", "sfa_rope.hip", "sfa_format.hip", "sfa_noalloc.hip", "sfa_capi.cpp"]
ARCH = "gfx950"


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _flags():
    return ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
            # no packed fp32 VALU instructions in device code
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", os.path.join(ROOT, "include"), "-Wno-unused-command-line-argument"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [_hipcc()] + _flags() + ["-c", os.path.join(CSRC, src), "-o", obj]
    _run(cmd, "compile")
    return obj


def _run(cmd, what: str):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")


def _build_binding() -> None:
    import torch
    troot = os.path.dirname(torch.__file__)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(_hipcc())))
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-I", os.path.join(troot, "include"),
          "-I", os.path.join(troot, "include", "torch", "csrc", "api", "include"),
          "-I", sysconfig.get_paths()["include"], "-I", os.path.join(rocm, "include"),
          os.path.join(CSRC, "sfa_binding.cpp"), "-o", BINDING + ".tmp",
          "-L", os.path.join(troot, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"], "binding")
    os.replace(BINDING + ".tmp", BINDING)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        binding = ex.submit(_build_binding)
        objs = list(ex.map(_compile, SOURCES))
        binding.result()
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    _run(cmd, "link")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB} and {BINDING}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
