"""Builds libmoegps.so (the C-ABI library, sm_100a only) in-tree with nvcc, and with the host compiler the Python module
_marshal (argument checks of the training step's calls, csrc/marshal.cpp)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libmoegps.so")
MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")
MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ["api.cu", "route.cu", "histogram.cu", "plan.cu", "pack.cu", "dispatch.cu", "expert_ffn.cu", "combine.cu",
           "predictor.cu", "selftest.cu", "expert_ffn_backward.cu", "shuffle_backward.cu", "route_backward.cu",
           "experts4.cu", "expert_ffn4.cu"]
HEADERS = ["common.cuh", "sm100.cuh", "route_epilogue.cuh", "slot_offsets.cuh", "grouped_gemm.cuh", "act8.cuh", "bf16x8.cuh",
           "route_backward.cuh", "mx4.cuh", "tile_sums.cuh"]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: libmoegps.so cannot be built")


def needs_build() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    built = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(ROOT, "include", "moegps.h")]
    return any(os.path.getmtime(d) > built for d in deps)


def marshal_marker() -> str:
    """What a _marshal of this torch carries (its attribute `built_for`): it reads torch's C++ objects directly."""
    import torch
    return f"moegps _marshal for torch {torch.__version__}"


def _marshal_is_current() -> bool:
    if not os.path.exists(MARSHAL_PATH) or os.path.getmtime(MARSHAL_SOURCE) > os.path.getmtime(MARSHAL_PATH):
        return False
    with open(MARSHAL_PATH, "rb") as f:
        return marshal_marker().encode() in f.read()


def build_marshal(force: bool = False) -> str:
    """Compile _marshal against the installed torch; returns its path."""
    if not force and _marshal_is_current():
        return MARSHAL_PATH
    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    cmd = [
        "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", f'-DMOEGPS_BUILT_FOR="{marshal_marker()}"',
        "-I", os.path.join(home, "include"), "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"),
        "-I", cuda, "-I", sysconfig.get_path("include"), MARSHAL_SOURCE,
        "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-o", MARSHAL_PATH + ".tmp",
    ]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
        raise RuntimeError("g++ failed building _marshal")
    os.replace(MARSHAL_PATH + ".tmp", MARSHAL_PATH)
    return MARSHAL_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu of the library for sm_100a into one shared object (and _marshal); returns its path.

    _marshal is optional (binding.py makes the same checks): where it cannot be compiled that is said, and no old one stays."""
    if force or needs_build():
        _build_library(verbose)
    try:
        build_marshal(force)
    except (RuntimeError, OSError) as e:
        sys.stderr.write(f"_marshal was not built ({e}): tensors are checked in Python, some microseconds a call slower\n")
        if os.path.exists(MARSHAL_PATH):
            os.remove(MARSHAL_PATH)
    return LIB_PATH


def _build_library(verbose: bool) -> None:
    cmd = [
        _nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
        "--threads", "8", "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    ]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES] + ["-o", LIB_PATH + ".tmp"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
        raise RuntimeError("nvcc failed building libmoegps.so")
    if verbose:
        sys.stderr.write(proc.stdout + proc.stderr)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
