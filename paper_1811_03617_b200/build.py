"""Builds libgvq.so (the CUDA kernels and their C ABI) in-tree with nvcc for sm_100a, and with the C++ compiler a module that is the short way
to some of its entry points from Python.  The module needs Python's and torch's headers and fits one version of either, which its file's name
says; without it gvq.py calls the library through ctypes."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import warnings
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libgvq.so"

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "8"]


def sources():
    return sorted(CSRC.glob("*.cu"))


def binding_path() -> Path:
    """The module for this Python and this torch."""
    import sysconfig

    import torch
    return PKG / f"_binding.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}.so"


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


def _older(out: Path, deps) -> bool:
    return not out.exists() or any(p.stat().st_mtime > out.stat().st_mtime for p in deps)


def _headers() -> list:
    return list((ROOT / "include").glob("*.h"))


def _stale() -> bool:
    return _older(LIB, [*sources(), *CSRC.glob("*.h"), *CSRC.glob("*.cuh"), *_headers()])


def _stale_binding() -> bool:
    return _older(binding_path(), [*CSRC.glob("*.cpp"), *_headers()])


class _Compilation:
    """A compiler at work on a file that takes its name once it is whole; a failure leaves nothing."""

    def __init__(self, out: Path, command):
        self.out, self.tmp = out, out.with_name(f"{out.name}.tmp{os.getpid()}")
        self.process = subprocess.Popen(command(self.tmp))

    def wait(self) -> None:
        try:
            if self.process.wait():
                raise subprocess.CalledProcessError(self.process.returncode, self.process.args)
            os.replace(self.tmp, self.out)
        finally:
            self.tmp.unlink(missing_ok=True)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every .cu under csrc/ into paper_1811_03617_b200/libgvq.so, and binding.cpp into the module beside it.  The library is wanted;
    a module that cannot be built (no headers) is a warning."""
    def library(tmp):
        nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
        return [nvcc, *NVCC_FLAGS, f"-I{ROOT / 'include'}", f"-I{CSRC}", *(["-Xptxas", "-v"] if verbose else []), *map(str, sources()),
                "-o", str(tmp), "-lcuda"]
    binding, problem = None, None
    if force or _stale_binding():
        try:
            binding = _Compilation(binding_path(), _binding_command)
        except OSError as e:
            problem = e
    try:
        if force or _stale():
            _Compilation(LIB, library).wait()
    finally:
        if binding is not None:
            try:
                binding.wait()
            except subprocess.CalledProcessError as e:
                problem = e
    if problem is not None:
        warnings.warn(f"{binding_path().name} was not built ({problem}): gvq.py calls the library through ctypes, at some microseconds a call",
                      RuntimeWarning, stacklevel=2)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
