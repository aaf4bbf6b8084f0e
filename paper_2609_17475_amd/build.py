"""Build libjfkv.so in-tree with hipcc for gfx950.

Each source is compiled to an object in ``paper_2609_17475_amd/_build`` (in
parallel), then linked into ``paper_2609_17475_amd/libjfkv.so``.  Packed-fp32
VALU forms are disabled for all device code.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libjfkv.so")
ARCH = os.environ.get("JFKV_ARCH", "gfx950")

SOURCES = ["jfkv_host.cpp", "quantize.hip", "decode.hip", "prefill.hip", "tq4.hip",
           "tq4_decode.hip", "reconstruct.hip", "pages.hip", "calib.hip", "kv8_host.cpp",
           "kv8_append.hip", "kv8_decode.hip", "kv8_prefill.hip", "kv8_evict.hip", "rope_host.cpp", "rope.hip",
           "kv8_shared_host.cpp", "kv8_shared.hip"]

COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
          "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
DEVICE = ["--offload-arch=" + ARCH, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-munsafe-fp-atomics"]
# Per-source device flags.  decode.hip: matrix-core results stay in ordinary
# VGPRs (its rare rescale multiplies them on the VALU; with accumulation
# registers the compiler copies them out and back around every row); the
# decodes over the 8-bit cache likewise.
EXTRA = {"decode.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "kv8_decode.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "kv8_shared.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def hipcc() -> str:
    p = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    return p


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    path = os.path.join(CSRC, src)
    cmd = [hipcc(), *COMMON]
    if src.endswith(".hip"):
        cmd += ["-x", "hip", *DEVICE, *EXTRA.get(src, [])]
    else:
        cmd += ["-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include"]
    cmd += ["-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("compile failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc(), "--offload-arch=" + ARCH, "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
