"""Builds librag_attn.so (gfx950) in-tree with hipcc.

    python -m paper_2412_10543_amd.build        # or __graft_entry__.build()
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBRARY = os.path.join(PKG, "librag_attn.so")
OBJDIR = os.path.join(PKG, "_build")

ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Packed fp32 VALU instructions are kept out of every kernel.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", INCLUDE, "-I", CSRC,
          "-Wall", "-Wno-unused-result"]

# Per-source device flags.  The int4 GEMM keeps its MFMA accumulators in
# ordinary VGPRs, where the per-group rescaling (a VALU multiply) can reach
# them without AGPR copies.
SOURCE_FLAGS = {"awq_gemm.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}
SOURCES = ["kernels.hip", "kv_cache.hip", "awq_gemm.hip", "decode_scratch.hip", "tree_decode.hip",
           "ranges_prefill.hip", "kv_pages.hip", "rope_write.hip", "kv4_read.hip", "kv4_decode.hip",
           "draft_verify.hip", "api.cpp", "awq_api.cpp", "draft_api.cpp", "serve_api.cpp",
           "planner.cpp"]
HEADERS = ["common.h", "prefill_tile.h", "decode_unit.h", "launch.h", "errors.h", "awq.h",
           "checks.h", "draft.h", "masked_tile.h", "kv4.h", "serve.h"]


PROBES = os.path.join(PKG, "libceiling_probes.so")


def build_probes(verbose: bool = False) -> str:
    """The hardware ceiling probes (measurement only, not the method)."""
    os.makedirs(OBJDIR, exist_ok=True)
    obj = os.path.join(OBJDIR, "ceiling_probes.o")
    cmd = [HIPCC, *COMMON, *DEVICE_FLAGS, "-x", "hip", "-c",
           os.path.join(CSRC, "ceiling_probes.hip"), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, stderr=None if verbose else subprocess.PIPE)
    tmp = PROBES + ".tmp"
    subprocess.run([HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, obj], check=True)
    os.replace(tmp, PROBES)
    return PROBES


MARSHAL = os.path.join(PKG, "_marshal.so")


def build_marshal(verbose: bool = False) -> str:
    """The binding's checks of tensors (host code against torch's headers)."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    tmp = MARSHAL + ".tmp"
    cmd = [HIPCC, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared",
           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{p}" for p in include_paths("cuda")), "-I" + sysconfig.get_paths()["include"],
           os.path.join(CSRC, "marshal.cpp"), "-o", tmp,
           *(f"-L{p}" for p in library_paths("cuda")), "-ltorch_python", "-ltorch", "-ltorch_cpu",
           "-lc10", "-lc10_hip"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, stderr=None if verbose else subprocess.PIPE)
    os.replace(tmp, MARSHAL)
    return MARSHAL


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    objs = []
    for src in SOURCES:
        obj = os.path.join(OBJDIR, os.path.splitext(src)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else ["-x", "hip"]
        cmd = [HIPCC, *COMMON, *DEVICE_FLAGS, *SOURCE_FLAGS.get(src, []), *lang, "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True, stderr=None if verbose else subprocess.PIPE)
        objs.append(obj)
    tmp = LIBRARY + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIBRARY)
    build_probes(verbose)
    if importlib.util.find_spec("torch") is not None:   # (without it there are no tensors to check)
        build_marshal(verbose)
    return LIBRARY


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIBRARY)
