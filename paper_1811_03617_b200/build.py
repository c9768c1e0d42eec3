"""Builds libgvq.so (the CUDA kernels and their C ABI) in-tree with nvcc for sm_100a, and _binding.so (the short way to some of its entry
points from Python) with the C++ compiler."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libgvq.so"
BINDING = PKG / "_binding.so"

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "8"]


def sources():
    return sorted(CSRC.glob("*.cu"))


def _binding_command(out) -> list:
    import sysconfig

    import torch
    t = Path(torch.__file__).resolve().parent
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    cuda = Path(nvcc).resolve().parent.parent / "include"
    return [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-shared", "-fPIC",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{sysconfig.get_paths()['include']}", f"-I{t / 'include'}",
            f"-I{t / 'include/torch/csrc/api/include'}", f"-I{cuda}", f"-I{ROOT / 'include'}", str(CSRC / "binding.cpp"), "-o", str(out),
            f"-L{t / 'lib'}", "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]


def _stale() -> bool:
    if not LIB.exists() or not BINDING.exists():
        return True
    t = min(LIB.stat().st_mtime, BINDING.stat().st_mtime)
    deps = list(CSRC.glob("*.cu")) + list(CSRC.glob("*.h")) + list(CSRC.glob("*.cuh")) + list(CSRC.glob("*.cpp")) + list((ROOT / "include").glob("*.h"))
    return any(p.stat().st_mtime > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every .cu under csrc/ into paper_1811_03617_b200/libgvq.so, and binding.cpp into _binding.so."""
    if not force and not _stale():
        return LIB
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    tmp = LIB.with_suffix(f".so.tmp{os.getpid()}")
    cmd = [nvcc, *NVCC_FLAGS, f"-I{ROOT / 'include'}", f"-I{CSRC}"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [str(s) for s in sources()] + ["-o", str(tmp), "-lcuda"]
    tmp_binding = BINDING.with_suffix(f".so.tmp{os.getpid()}")
    binding = subprocess.Popen(_binding_command(tmp_binding))
    try:
        try:
            subprocess.run(cmd, check=True)
        finally:
            status = binding.wait()
        if status:
            raise subprocess.CalledProcessError(status, binding.args)
        os.replace(tmp, LIB)
        os.replace(tmp_binding, BINDING)
    finally:
        for path in (tmp, tmp_binding):      # (what a failure leaves)
            path.unlink(missing_ok=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
