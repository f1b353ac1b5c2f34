"""Build libmalt.so (HIP, gfx950) in-tree with hipcc, and beside it the Python module
_malt.so (host code on torch's headers) and the matrix-core calibration library
libmalt_calib.so.

Usage: python -m paper_2608_05088_amd.build [-v]
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "lib", "libmalt.so")
BINDING_LIB = os.path.join(PKG, "lib", "_malt.so")
CALIB = os.path.join(PKG, "calib")
CALIB_LIB = os.path.join(PKG, "lib", "libmalt_calib.so")
SOURCES = ["malt_api.hip", "elementwise.hip", "ns_sym.hip", "ns_update.hip", "ns_mid.hip", "small_ns.hip",
           "embed.hip", "distill.hip", "block_quant.hip", "block_matmul.hip", "block_linear.hip",
           "ops_api.hip", "adamw.hip", "norm.hip", "head.hip", "head_rows.hip", "model_api.hip"]
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm toolchain required to build libmalt)")


def build_cmd(out: str = LIB) -> list:
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
            # Packed-fp32 VALU forms are disabled for all device code.
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            *[os.path.join(CSRC, s) for s in SOURCES],
            "-o", out]


def binding_cmd(out: str = BINDING_LIB) -> list:
    import sysconfig
    from torch.utils import cpp_extension
    torch_lib = cpp_extension.library_paths()[0]
    return [hipcc(), "-x", "hip", "--cuda-host-only", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            "-Wall", "-Wno-unused-function", "-Wno-deprecated-declarations", "-Wno-unused-result",
            *[f"-I{p}" for p in cpp_extension.include_paths()], "-I", sysconfig.get_paths()["include"],
            os.path.join(CSRC, "binding.cpp"), "-L", os.path.dirname(LIB), "-l:libmalt.so", "-Wl,-rpath,$ORIGIN",
            "-L", torch_lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip", "-o", out]


def calib_cmd(out: str = CALIB_LIB) -> list:
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", os.path.join(CALIB, "mfma_ceiling.hip"), "-o", out]


def _compile(cmd: list, lib: str, what: str, verbose: bool) -> None:
    tmp = cmd[-1]
    if verbose:
        print(" ".join(cmd), flush=True)
    proc = subprocess.run(cmd, cwd=os.path.dirname(lib), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # hipcc's host pass does not know the packed-fp32 feature; that note is harmless.
    out = "\n".join(l for l in proc.stdout.splitlines() if "packed-fp32-ops" not in l)
    if proc.returncode != 0:
        raise RuntimeError(f"{what} build failed ({proc.returncode}):\n{out}")
    if verbose and out.strip():
        print(out)
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    """Compile every HIP source of the package into libmalt.so, the host side of the
    operators into _malt.so and the matrix-core calibration into libmalt_calib.so (always
    rebuilds)."""
    os.makedirs(os.path.dirname(LIB), exist_ok=True)
    _compile(build_cmd(LIB + ".tmp"), LIB, "libmalt", verbose)
    _compile(binding_cmd(BINDING_LIB + ".tmp"), BINDING_LIB, "_malt", verbose)
    _compile(calib_cmd(CALIB_LIB + ".tmp"), CALIB_LIB, "libmalt_calib", verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
