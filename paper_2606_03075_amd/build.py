"""Build libtgvkv.so for gfx950 in-tree with hipcc (no torch, no JIT cache).

python -m paper_2606_03075_amd.build   (or __graft_entry__.build())
"""

from __future__ import annotations

import concurrent.futures as fut
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build", "tgvkv")
LIB = os.path.join(PKG, "libtgvkv.so")

HIP_SOURCES = ["score.hip", "budget.hip", "select.hip", "compact.hip", "decode.hip", "pages.hip", "quant.hip", "chunk.hip",
               "ceiling.hip"]
CXX_SOURCES = ["api.cpp"]
ARCH = "gfx950"


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def common_flags():
    return ["-O3", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function", f"-I{INCLUDE}", f"-I{CSRC}"]


# Sources whose kernels run with the IEEE mode bit off (see device_flags).
NO_IEEE_SOURCES = ("score.hip",)


def device_flags(src=None):
    # Packed-fp32 VALU forms are disabled for all device code.  MFMA results are
    # kept in ordinary VGPRs (gfx950 allows it): the accumulator-register form
    # costs a v_accvgpr_read per result register before the softmax arithmetic.
    flags = [f"--offload-arch={ARCH}", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-munsafe-fp-atomics", "-mllvm", "-amdgpu-mfma-vgpr-form"]
    # The scoring kernels create no NaNs (every -inf - -inf is guarded), so they run
    # with the IEEE mode bit off: with it on, each MFMA result needs a quieting
    # v_max x, x before a running max can use it (64 of the 540 VALU instructions
    # per tile of the statistics sweep); for finite values the results are the
    # same bits.  (Elsewhere the change cost occupancy and saved nothing.)
    if src in NO_IEEE_SOURCES:
        flags += ["-fno-honor-nans", "-mno-amdgpu-ieee"]
    return flags


def _compile(src: str, verbose: bool) -> str:
    path = os.path.join(CSRC, src)
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc()] + common_flags()
    if src.endswith(".hip"):
        cmd += device_flags(src) + ["-x", "hip"]
    else:
        cmd += ["-D__HIP_PLATFORM_AMD__"]
    cmd += ["-c", path, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {src}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every source for gfx950 and link libtgvkv.so; returns the library path."""
    os.makedirs(BUILD, exist_ok=True)
    with fut.ThreadPoolExecutor(max(1, min(jobs, 16))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), HIP_SOURCES + CXX_SOURCES))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


SAN_BUILD = os.path.join(ROOT, "_build", "tgvkv_san")
SAN_LIB = os.path.join(SAN_BUILD, "libtgvkv_san.so")
SAN_FLAGS = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g"]


def build_sanitized(verbose: bool = False) -> str:
    """A host-sanitized copy of the library for CPU tests of the C ABI: api.cpp (argument
    validation, workspace layout, launch set-up) built by g++ with AddressSanitizer and
    UndefinedBehaviorSanitizer, linked with the unsanitized device objects of build().
    Load it with libasan / libubsan preloaded (the Python interpreter is not instrumented).
    Returns the library path (under _build/, never shipped)."""
    os.makedirs(SAN_BUILD, exist_ok=True)
    dev_objs = [os.path.join(BUILD, os.path.splitext(src)[0] + ".o") for src in HIP_SOURCES]
    if not all(os.path.exists(o) for o in dev_objs):
        build(verbose)
    obj = os.path.join(SAN_BUILD, "api_san.o")
    cmd = ["g++", "-O1", "-fPIC", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__", f"-I{INCLUDE}", f"-I{CSRC}",
           "-I/opt/rocm/include"] + SAN_FLAGS + ["-c", os.path.join(CSRC, "api.cpp"), "-o", obj]
    for c in (cmd, ["g++", "-shared", "-o", SAN_LIB, obj] + dev_objs + SAN_FLAGS[:1] +
              ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"]):
        if verbose:
            print(" ".join(c), flush=True)
        r = subprocess.run(c, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"sanitized build failed\n{r.stdout}\n{r.stderr}")
    return SAN_LIB


if __name__ == "__main__":
    if "--sanitize" in sys.argv:
        print(build_sanitized(verbose="-v" in sys.argv))
    else:
        print(build(verbose="-v" in sys.argv))
