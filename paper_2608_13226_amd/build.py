"""Build libcoverprune.so for gfx950 with hipcc, in-tree.

Each .hip source under csrc/ is compiled to an object in parallel, then the
objects are linked into paper_2608_13226_amd/libcoverprune.so.  The compiled
half of the serving operators' binding (csrc/binding.cpp, host code against
torch's headers) is built beside it as _serving.so.  Run as
``python -m paper_2608_13226_amd.build``.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libcoverprune.so")
BINDING = os.path.join(HERE, "_serving.so")
ARCH = "gfx950"

# Packed fp32 instructions are disabled for all device code.
FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-function"]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    cmd = [hipcc(), *FLAGS, "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{res.stderr}")
    noise = [ln for ln in res.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip()]
    if noise:
        sys.stderr.write("\n".join(noise) + "\n")
    return obj


def _compile_binding() -> str:
    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(OBJ, "binding.cpp.o")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-isystem", os.path.join(root, "include"),
           "-isystem", sysconfig.get_paths()["include"], "-c", os.path.join(CSRC, "binding.cpp"), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed on binding.cpp:\n{res.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    """Against the library beside it and the torch that the process has loaded."""
    import torch
    tmp = BINDING + ".tmp"
    cmd = ["g++", "-shared", obj, "-o", tmp, "-L", os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python",
           "-ltorch_cpu", "-lc10", "-L", HERE, "-lcoverprune", "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link of the binding failed:\n{res.stderr}")
    os.replace(tmp, BINDING)


def build(jobs: int = 8) -> str:
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with ThreadPoolExecutor(max_workers=max(1, min(jobs, len(srcs) + 1))) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, LIB)
    _link_binding(binding.result())
    return LIB


if __name__ == "__main__":
    print(build())
