"""Builds libspconv.so (all HIP sources, gfx950) in the package directory."""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libspconv.so")
TORCH_OPS = os.path.join(HERE, "_torch_ops.so")  # the transformer operators' binding (host code only)
SOURCES = ["api.hip", "scan.hip", "map_kernels.hip", "gmas_kernels.hip", "gemm_mfma.hip", "conv_small.hip",
           "norm.hip", "linear8.hip", "attention.hip", "attention_tile.hip", "attention_rows.hip", "attention_pages.hip",
           "attention_pages8.hip", "attention_small.hip", "attention_small8.hip", "rotate.hip", "cache.hip"]
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result",
    # packed FP32 instructions stay off (they are not used by any kernel here)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def _torch_ops() -> str:
    """The binding against the installed torch (its folder is found without importing it)."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("the torch binding (_torch_ops.so) needs torch and its headers")
    torch = os.path.dirname(spec.origin)
    tmp = TORCH_OPS + ".tmp"
    cmd = [HIPCC, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-DUSE_ROCM", "-D__HIP_PLATFORM_AMD__",
           "-I", INCLUDE, "-isystem", os.path.join(torch, "include"), "-isystem", "/opt/rocm/include",
           "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "torch_ops.cpp"), "-o", tmp,
           "-L", os.path.join(torch, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for torch_ops.cpp:\n{r.stderr}")
    os.replace(tmp, TORCH_OPS)
    return TORCH_OPS


def build(jobs: int = 8) -> str:
    """Compile every HIP source for gfx950 and link libspconv.so, and the torch binding (always rebuilds).
    A binding that does not compile raises once the library, which needs no torch, is there."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=max(1, min(jobs, len(SOURCES)))) as ex:
        binding = ex.submit(_torch_ops)
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    binding.result()
    return LIB


if __name__ == "__main__":
    print(build())
