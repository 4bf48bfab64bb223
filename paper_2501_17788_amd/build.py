"""Build libwarp.so (the HIP kernels, gfx950 only) in-tree with hipcc, and _encoder.so, the native Python
binding of the token encoder's operators, with g++ against torch's headers."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")  # the search engine
CSRC_ENCODER = os.path.join(PKG, "csrc_encoder")  # the token encoder's operators
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libwarp.so")
BINDING = os.path.join(PKG, "_encoder.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result",
    # no packed-FP32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC, "-I", CSRC_ENCODER,
]


def sources() -> list[str]:
    return sorted(f for d in (CSRC, CSRC_ENCODER) for f in glob.glob(os.path.join(d, "*.hip")))


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [HIPCC, *FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _compile_binding() -> str | None:
    """The object of the native binding; None without torch, which the binding is for."""
    try:
        import torch
    except ImportError:
        return None
    at = os.path.dirname(torch.__file__)
    obj = os.path.join(BUILD, "encoder_binding.cpp.o")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           "-DTORCH_EXTENSION_NAME=_encoder", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", INCLUDE, "-isystem", os.path.join(at, "include"),
           "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
           "-isystem", sysconfig.get_paths()["include"],
           "-c", os.path.join(CSRC_ENCODER, "encoder_binding.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on encoder_binding.cpp:\n{r.stdout}\n{r.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    import torch

    tmp = BINDING + ".tmp"
    # libwarp.so and torch's libraries are loaded before the binding; libwarp.so lies beside it
    cmd = ["g++", "-shared", obj, "-o", tmp, "-L", os.path.join(os.path.dirname(torch.__file__), "lib"),
           "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_hip", "-L", PKG, "-l:libwarp.so",
           "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link of the binding failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)


def build(jobs: int | None = None) -> str:
    """Compile every HIP source for gfx950 and link libwarp.so, then the binding (always rebuilds)."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = sources()
    jobs = jobs or min(8, len(srcs) + 1)
    with ThreadPoolExecutor(jobs) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,--no-undefined", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    obj = binding.result()  # after the library, which does without it
    if obj:
        _link_binding(obj)
    return LIB


if __name__ == "__main__":
    print(build(int(sys.argv[1]) if len(sys.argv) > 1 else None))
