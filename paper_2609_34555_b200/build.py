"""Builds libpulseinfer_b200.so (sm_100a only) in-tree with nvcc, and _front, the Python module that checks
the tensors of the calls on the 4-bit and 8-bit paths and of the attention over prompts, with g++ against the installed
torch.  Only those calls need the module.

    python -m paper_2609_34555_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
INCLUDE = PKG.parent / "include"
LIB = PKG / "libpulseinfer_b200.so"

SOURCES = ["pi_api.cu", "pi_score_select.cu", "pi_select_diff.cu", "pi_diff_misses.cu", "pi_recall.cu", "pi_attn.cu", "pi_attn_headmajor.cu",
           "pi_helpers.cu", "pi_append.cu", "pi_api_kv4.cu", "pi_kv4.cu", "pi_rope.cu", "pi_pages.cu", "pi_attn_kv4.cu",
           "pi_api_prompt.cu", "pi_prompt_attn.cu", "pi_api_kv8.cu", "pi_kv8.cu", "pi_append_kv8.cu", "pi_attn_kv8.cu"]


def sources() -> list[Path]:
    return [CSRC / s for s in SOURCES if (CSRC / s).exists()]


def _stale() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    deps = sources() + list(CSRC.glob("*.cuh")) + list(INCLUDE.glob("*.h"))
    return any(d.stat().st_mtime > t for d in deps)


def front_path() -> Path:
    """The module reads torch's tensors as its headers lay them out: one file for each torch, C++ ABI and Python."""
    import torch
    return PKG / f"_front.torch-{torch.__version__}.abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}{sysconfig.get_config_var('EXT_SUFFIX') or '.so'}"


def build_front(force: bool = False) -> Path:
    front = front_path()
    deps = [CSRC / "front.cpp"] + list(INCLUDE.glob("*.h"))
    if not force and front.exists() and all(d.stat().st_mtime <= front.stat().st_mtime for d in deps):
        return front
    import torch
    root = Path(torch.__file__).resolve().parent
    tmp = front.with_suffix(f".tmp{os.getpid()}.so")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                           f"-I{INCLUDE}", f"-I{sysconfig.get_paths()['include']}", f"-I{root / 'include'}", f"-I{root / 'include' / 'torch' / 'csrc' / 'api' / 'include'}",
                           "-o", str(tmp), str(CSRC / "front.cpp"), f"-L{root / 'lib'}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, front)
    return front


def build(force: bool = False, verbose: bool = False) -> Path:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB.with_suffix(f".tmp{os.getpid()}.so")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", f"-I{INCLUDE}", f"-I{CSRC}",
           "-o", str(tmp)] + [str(s) for s in sources()]
    cmd[1:1] = os.environ.get("PI_NVCC_FLAGS", "").split()       # extra flags for experiments (-D..., -Xptxas=-v)
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
    print(build_front(force="--force" in sys.argv))
