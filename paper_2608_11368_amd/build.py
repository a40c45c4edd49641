"""Build libpair.so (HIP, gfx950) in-tree with hipcc.

Usage: python -m paper_2608_11368_amd.build
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpair.so")
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


def build(verbose: bool = False, out: str = LIB, build_dir: str = BUILD,
          host_flags=(), link_flags=()) -> str:
    """Compile every source and link the shared library at `out`.
    `host_flags` apply to the host-side compilation only (each is passed
    after -Xarch_host), e.g. a sanitizer for the host argument checks."""
    os.makedirs(build_dir, exist_ok=True)
    extra = [x for f in host_flags for x in ("-Xarch_host", f)]
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda src: _compile(src, build_dir, extra), SOURCES))
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
