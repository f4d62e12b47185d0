"""Build libff.so (HIP, gfx950) and the module _calls (the binding's part in C++) in-tree.

    python -m paper_2203_00854_amd.build

hipcc cross-compiles for gfx950 without a GPU.  Objects go to _build/, the library to
paper_2203_00854_amd/libff.so, the module, of one interpreter's version, beside it (git-ignored; they travel with the source tree to the GPU machine).
The library needs hipcc alone.  Where g++, torch or the interpreter's headers are missing the module is left out, and with it the Python entry points of the training operators.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libff.so")
CALLS = os.path.join(PKG, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=fast",
    "-Wall", "-Wno-unused-function",
    # the direct-to-LDS loads of the GEMM set M0 in inline assembly and name it as clobbered; the
    # compiler remarks that M0 is a reserved register (k_gemm has no other user of M0)
    "-Wno-inline-asm",
    # packed-FP32 VALU forms are switched off for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix-core accumulators live in ordinary VGPRs: the softmax works on them directly,
    # so the AGPR form would cost a register move per element and tile
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]
# the optimiser's states are the same to the last bit as its formulas evaluated one rounded operation at a time
# (8-bit codes would show a difference as a whole step), so none of its products is fused with a sum
SOURCE_FLAGS = {"ff_adamw.hip": ["-ffp-contract=off"]}


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(os.path.basename(src), []), "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l and l.strip())
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    if err:
        sys.stderr.write(err + "\n")
    return obj


def _build_calls() -> str:
    """ff_calls.cpp, host code: a CPython module on libff.so and torch's libraries.  What is missing for it, or ""."""
    for old in (CALLS, os.path.join(PKG, "_calls.so")):          # (the latter: without an interpreter's version, as it was once named)
        if os.path.exists(old):
            os.remove(old)
    compiler = shutil.which("g++")
    if not compiler:
        return "g++"
    try:
        import torch
    except ImportError:
        return "torch"
    home = os.path.dirname(torch.__file__)
    for header in (os.path.join(sysconfig.get_paths()["include"], "Python.h"), os.path.join(home, "include", "ATen", "ATen.h")):
        if not os.path.exists(header):
            return header
    cmd = [compiler, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(home, "include"),
           "-isystem", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"), os.path.join(CSRC, "ff_calls.cpp"), "-o", CALLS,
           "-L", PKG, "-l:libff.so", "-L", os.path.join(home, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for ff_calls.cpp:\n" + r.stderr)
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    return ""


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    missing = _build_calls()
    if missing:
        print(f"without {missing}: {os.path.basename(CALLS)} is left out, and with it the Python entry points of the training operators")
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources" + ("" if missing else f", {CALLS}"))
    return LIB


if __name__ == "__main__":
    build()
