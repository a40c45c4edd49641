"""Build libpair.so (HIP, gfx950) in-tree with hipcc, and the binding's reader of
tensor lists (_tensors.so, host only) with g++ against the installed torch.

Usage: python -m paper_2608_11368_amd.build
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpair.so")
TENSORS = os.path.join(HERE, "_tensors.so")
SOURCES = ["api.hip", "design.hip", "coeffs.hip", "wgrad.hip", "audit.hip", "exact.hip", "alloc.hip",
           "cps.hip", "noalloc.hip", "clip.hip", "pages.hip", "attn.hip", "attn_rows.hip",
           "attn_tiles.hip"]
ARCH = "gfx950"

# Packed fp32 VALU ops are kept off in all device code.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                # matrix-core results in ordinary VGPRs: the epilogue reads them directly
                "-mllvm", "-amdgpu-mfma-vgpr-form"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Wall",
          "-Wno-unused-command-line-argument"] + DEVICE_FLAGS


def _hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def _compile(src: str, build_dir: str = BUILD, extra=()) -> str:
    obj = os.path.join(build_dir, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), *COMMON, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        print(err, file=sys.stderr)
    return obj


def build_tensors(out: str = TENSORS) -> str:
    """Compile csrc/tensors.cpp as the extension module at `out`."""
    import torch

    root = os.path.dirname(torch.__file__)
    tmp = out + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I" + sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
           "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(CSRC, "tensors.cpp"), "-o", tmp, "-L" + os.path.join(root, "lib"),
           "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed for tensors.cpp:\n{res.stderr}")
    os.replace(tmp, out)
    return out


def build(verbose: bool = False, out: str = LIB, build_dir: str = BUILD,
          host_flags=(), link_flags=()) -> str:
    """Compile every source and link the shared library at `out` (the default one
    with the binding's extension module beside it).
    `host_flags` apply to the host-side compilation only (each is passed
    after -Xarch_host), e.g. a sanitizer for the host argument checks."""
    os.makedirs(build_dir, exist_ok=True)
    extra = [x for f in host_flags for x in ("-Xarch_host", f)]
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        tensors = ex.submit(build_tensors) if out == LIB else None
        objs = list(ex.map(lambda src: _compile(src, build_dir, extra), SOURCES))
        if tensors is not None:
            tensors.result()
    tmp = out + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs, *link_flags]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, out)
    if verbose:
        print(f"built {out}")
    return out


if __name__ == "__main__":
    build(verbose=True)
