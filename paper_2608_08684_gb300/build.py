"""In-tree build of libripple.so (CUDA kernels for sm_103a + the host C allocator) and of
the extension module _binding.<versions>.so (argument marshalling of the per-layer calls,
against the installed Python and PyTorch, which its name tells).

Each translation unit is compiled in parallel with nvcc (CUDA) or gcc (C), then
linked with nvcc into paper_2608_08684_gb300/libripple.so. The build is skipped
when the library is newer than every source and header.

build_library(checked=True) builds libripple_checked.so from the same sources
with RIPPLE_CHECKED defined: every guarded global access in the kernels tests
its offset against its buffer's extent and reports RIPPLE_EBOUNDS in the
call's status word instead of going out of bounds (the bounds-check build that
stands in for a memory checker; the binding loads it when RIPPLE_CHECKED=1 is
set in the environment).
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libripple.so")
BUILD_CHECKED = os.path.join(PKG, "_build_checked")
BINDING_SRC = os.path.join(CSRC, "binding.cpp")
LIB_CHECKED = os.path.join(PKG, "libripple_checked.so")

NVCC = os.environ.get("NVCC", "nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
                     "-Xcompiler", "-ffp-contract=off", "-I", INCLUDE, "-I", CSRC]
CC_FLAGS = ["-O2", "-std=c99", "-fPIC", "-ffp-contract=off", "-Wall", "-I", INCLUDE]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu"))) + sorted(glob.glob(os.path.join(CSRC, "*.c")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))


def _stale(lib: str, deps=None) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(p) > t for p in deps or _deps())


def _compile(src: str, extra: list, build_dir: str) -> str:
    obj = os.path.join(build_dir, os.path.basename(src) + ".o")
    if src.endswith(".cu"):
        cmd = [NVCC] + NVCC_FLAGS + extra + ["-c", src, "-o", obj]
    else:
        cmd = [os.environ.get("CC", "gcc")] + CC_FLAGS + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def binding_path() -> str:
    """The extension module for the running Python and PyTorch. It reads tensors through
    accessors compiled into it, so one built for another version must not be loaded: the name
    holds Python's ABI and PyTorch's version, commit and C++ ABI."""
    import sysconfig

    import torch

    abi = sysconfig.get_config_var("SOABI") or "-".join(map(str, sys.version_info[:2]))
    commit = str(getattr(torch.version, "git_version", None))[:12]
    return os.path.join(PKG, f"_binding.{abi}.torch-{torch.__version__}-{commit}-"
                             f"cxx11abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}.so")


def build_binding(force: bool = False, verbose: bool = False) -> str:
    """Build the extension module if it is missing or older than its sources; return its
    path."""
    binding = binding_path()
    if not force and not _stale(binding, [BINDING_SRC, os.path.join(CSRC, "paged.cuh"),
                                          os.path.join(INCLUDE, "ripple.h")]):
        return binding
    import sysconfig

    import torch

    at = os.path.join(os.path.dirname(torch.__file__), "")
    nvcc = shutil.which(NVCC)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc))) if nvcc else "/usr/local/cuda"
    tmp = f"{binding}.{os.getpid()}.tmp"  # (processes may build at the same time)
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", BINDING_SRC,
           "-o", tmp, "-I", INCLUDE, "-I", at + "include",
           "-I", at + "include/torch/csrc/api/include", "-I", os.path.join(cuda, "include"),
           "-I", sysconfig.get_paths()["include"],
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-L", at + "lib", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda",
           f"-Wl,-rpath,{at}lib"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, binding)
    finally:
        if os.path.exists(tmp):
            os.remove(tmp)
    if verbose:
        print(f"built {binding}", file=sys.stderr)
    return binding


def build_library(force: bool = False, verbose: bool = False, extra_nvcc=(),
                  checked: bool = False) -> str:
    """Build libripple.so (libripple_checked.so with checked=True) if it is
    missing or older than its sources, and the binding's extension module; return the
    library's path. The library needs neither Python's headers nor PyTorch's: where the
    extension module cannot be built, this warns, and the calls that need it raise."""
    path = _build_library(force, verbose, extra_nvcc, checked)
    try:
        build_binding(force, verbose)
    except (RuntimeError, OSError, ImportError) as e:
        warnings.warn("the extension module could not be built: the paged calls and the log "
                      f"probabilities are not available from Python. {e}", RuntimeWarning, stacklevel=2)
    return path


def _build_library(force, verbose, extra_nvcc, checked) -> str:
    lib, build_dir = (LIB_CHECKED, BUILD_CHECKED) if checked else (LIB, BUILD)
    extra = list(extra_nvcc) + (["-DRIPPLE_CHECKED"] if checked else [])
    if not force and not _stale(lib):
        return lib
    os.makedirs(build_dir, exist_ok=True)
    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, extra, build_dir), srcs))
    tmp = lib + ".tmp"
    cmd = [NVCC] + ARCH + ["-shared", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)
    if verbose:
        print(f"built {lib}", file=sys.stderr)
    return lib


if __name__ == "__main__":
    build_library(force="--force" in sys.argv, verbose=True, checked="--checked" in sys.argv)
