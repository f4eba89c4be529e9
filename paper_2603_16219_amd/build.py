"""Compile the HIP library in-tree for gfx950 (hipcc cross-compiles without a GPU), and the binding's native wrappers."""
from __future__ import annotations

import hashlib
import os
import subprocess
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", n) for n in ("specsteer.hip", "split.hip")]
INCLUDE = os.path.join(_ROOT, "include")
LIBRARY = os.path.join(_PKG, "libspecsteer.so")
LOSS_SOURCES = [os.path.join(_PKG, "csrc", "loss", n) for n in ("loss.hip", "alternatives.hip")]
LOSS_LIBRARY = os.path.join(_PKG, "libspecsteer_loss.so")
TREE_SOURCES = [os.path.join(_PKG, "csrc", "tree", n) for n in ("attention.hip", "verify.hip", "commit.hip")]
TREE_LIBRARY = os.path.join(_PKG, "libspecsteer_tree.so")
CALLS_SOURCES = [os.path.join(_PKG, "csrc", "calls.cpp"), os.path.join(_PKG, "csrc", "calls_common.hpp"), os.path.join(_PKG, "csrc", "unbound.h"),
                 os.path.join(INCLUDE, "specsteer.h")]
LOSS_CALLS_SOURCES = [os.path.join(_PKG, "csrc", "loss", "loss_calls.cpp"), os.path.join(_PKG, "csrc", "calls_common.hpp"),
                      *(os.path.join(INCLUDE, n) for n in ("specsteer_alternatives.h", "specsteer_loss.h", "specsteer.h"))]
TREE_CALLS_SOURCES = [os.path.join(_PKG, "csrc", "tree", "tree_calls.cpp"), os.path.join(_PKG, "csrc", "calls_common.hpp"),
                      *(os.path.join(INCLUDE, n) for n in ("specsteer_tree.h", "specsteer.h"))]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950",
    # packed-fp32 instructions are switched off for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # The logit loads are 16 bytes wide on vector types that promise only element alignment (rows of an odd
    # vocabulary start anywhere).  This states to the compiler what the code relies on -- wide global loads at
    # any element-aligned address are legal on this target (the hardware's unaligned access mode, which the
    # ROCm kernel driver enables) -- instead of leaving it to the toolchain's default for the target.
    "-Xclang", "-target-feature", "-Xclang", "+unaligned-access-mode",
    "-shared", "-fPIC", "-Wl,-rpath,/opt/rocm/lib",
]


def _run(cmd: list, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n{proc.stdout}\n{proc.stderr}")


def build(verbose: bool = False) -> str:
    build_library(verbose)
    build_loss_library(verbose)
    build_tree_library(verbose)
    build_calls(verbose)
    build_loss_calls(verbose)
    build_tree_calls(verbose)
    return LIBRARY


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    _run([hipcc, *HIPCC_FLAGS, "-I", INCLUDE, "-o", LIBRARY, *SOURCES], verbose)
    return LIBRARY


def build_loss_library(verbose: bool = False) -> str:
    """The losses, a library of their own: who only verifies loads none of their kernels."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    _run([hipcc, *HIPCC_FLAGS, "-I", INCLUDE, "-o", LOSS_LIBRARY, *LOSS_SOURCES], verbose)
    return LOSS_LIBRARY


def build_tree_library(verbose: bool = False) -> str:
    """Trees of drafts, a library of their own too."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    _run([hipcc, *HIPCC_FLAGS, "-I", INCLUDE, "-o", TREE_LIBRARY, *TREE_SOURCES], verbose)
    return TREE_LIBRARY


def calls_path() -> str:
    """Where the native wrappers for this torch and these sources lie: what they are compiled against is in the name, so that one
    built for another torch, whose tensors may be laid out differently, or from other sources is never loaded."""
    return _calls_path("_calls", CALLS_SOURCES)


def loss_calls_path() -> str:
    """The same for those of the losses."""
    return _calls_path("_loss_calls", LOSS_CALLS_SOURCES)


def tree_calls_path() -> str:
    """The same for those of trees."""
    return _calls_path("_tree_calls", TREE_CALLS_SOURCES)


def _calls_path(name: str, sources: list) -> str:
    import torch

    h = hashlib.sha256(repr((torch.__version__, torch.version.git_version, torch._C._GLIBCXX_USE_CXX11_ABI)).encode())
    for path in sources:
        with open(path, "rb") as f:
            h.update(f.read())
    return os.path.join(_PKG, f"{name}-{h.hexdigest()[:16]}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_calls(verbose: bool = False) -> str:
    return _build_calls(calls_path(), CALLS_SOURCES[0], verbose)


def build_loss_calls(verbose: bool = False) -> str:
    return _build_calls(loss_calls_path(), LOSS_CALLS_SOURCES[0], verbose)


def build_tree_calls(verbose: bool = False) -> str:
    return _build_calls(tree_calls_path(), TREE_CALLS_SOURCES[0], verbose)


def _build_calls(path: str, source: str, verbose: bool) -> str:
    """The binding's native wrappers, host code against torch's headers and libraries.  Renamed into place, so that processes that
    build at the same time never load half a file."""
    import torch
    from torch.utils import cpp_extension

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    includes = [x for d in (INCLUDE, *cpp_extension.include_paths(), sysconfig.get_paths()["include"]) for x in ("-I", d)]
    part = f"{path}.{os.getpid()}"
    try:
        _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *includes, "-o", part, source,
              "-L", lib, "-lc10", "-ltorch_cpu", "-ltorch_python", f"-Wl,-rpath,{lib}"], verbose)
        os.replace(part, path)
    finally:
        if os.path.exists(part):
            os.remove(part)
    return path


if __name__ == "__main__":
    print(build(verbose=True))
