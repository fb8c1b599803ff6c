"""Compile the CUDA library in-tree: paper_2504_18454_b200/libpalsgd.so (sm_100a), and the native part of the
block operators' Python binding, paper_2504_18454_b200/_block.so (g++, against the installed torch).

nvcc cross-compiles without a GPU.  The runtime is linked statically, so the
library loads (and its pure-host entry points work) on a machine without a
driver; anything that touches the GPU then returns PALSGD_ECUDA.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
from pathlib import Path

HERE = Path(__file__).resolve().parent
CSRC = HERE / "csrc"
LIB = HERE / "libpalsgd.so"
EXT = HERE / "_block.so"
EXT_SOURCE = CSRC / "block_torch.cpp"
SOURCES = [CSRC / "palsgd_api.cu", CSRC / "palsgd_noalloc.cu", CSRC / "block_api.cu", CSRC / "block_norm_loss_api.cu"]
DEPS = sorted(CSRC.glob("*.cu*")) + sorted(CSRC.glob("*.h")) + sorted((HERE.parent / "include").glob("*.h")) + [Path(__file__)]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-std=c++17", "-lineinfo",
    "-fmad=false",                 # belt and braces: the kernels use *_rn intrinsics anyway
    "-Xcompiler", "-fPIC,-O2,-Wall",
    "-cudart", "static",
    "-shared",
]


def nvcc_path() -> str:
    return os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"


def needs_build() -> bool:
    if not LIB.exists():
        return True
    return LIB.stat().st_mtime < max(p.stat().st_mtime for p in DEPS)


def build_extension(force: bool = False) -> Path:
    """_block.so: it is bound to the loaded libpalsgd.so at run time and links torch only."""
    newest = max(p.stat().st_mtime for p in (EXT_SOURCE, *(HERE.parent / "include").glob("*.h"), Path(__file__)))
    if not force and EXT.exists() and EXT.stat().st_mtime >= newest:
        return EXT
    import sysconfig

    import torch
    home = Path(torch.__file__).resolve().parent
    cuda = Path(nvcc_path()).resolve().parent.parent
    tmp = HERE / f"_block.{os.getpid()}.tmp.so"
    subprocess.check_call([
        os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
        f"-I{home}/include", f"-I{home}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}",
        f"-I{cuda}/include", str(EXT_SOURCE), "-o", str(tmp),
        f"-L{home}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"])
    os.replace(tmp, EXT)
    return EXT


def build_library(force: bool = False, verbose: bool = False) -> Path:
    if not force and not needs_build():
        return LIB
    tmp = HERE / f"libpalsgd.{os.getpid()}.tmp.so"
    cmd = [nvcc_path(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *map(str, SOURCES), "-o", str(tmp)]
    env = dict(os.environ)
    env.pop("CC", None); env.pop("CXX", None)
    subprocess.check_call(cmd, env=env)
    os.replace(tmp, LIB)
    return LIB


def build(force: bool = False, verbose: bool = False) -> Path:
    """The library, then the block operators' binding where torch is installed: the library needs neither torch nor
    Python's headers, and the binding raises ImportError where it is missing."""
    build_library(force, verbose)
    if importlib.util.find_spec("torch"):
        build_extension(force)
    else:
        print("torch is not installed: the block operators' Python binding (_block.so) is not built", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
