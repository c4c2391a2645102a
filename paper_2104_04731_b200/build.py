"""Builds libb2conv.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SO = os.path.join(HERE, "libb2conv.so")
SO_DEBUG = os.path.join(HERE, "libb2conv_debug.so")  # -DB2C_DEBUG_BOUNDS: bounds-checked kernels, workspace guard bands
SOURCES = ["api.cpp", "planner.cpp", "tma.cpp", "layout.cu", "conv_mma.cu", "conv_mma_pair.cu", "mma_rate.cu", "conv_mma_window.cu", "conv_mma_plane.cu", "conv_mma_stream.cu",
           "fp8_api.cpp", "fp8_quantize.cu", "fp8_matmul.cu", "fp8_matmul_pair.cu", "route.cu",
           "fp4_api.cpp", "fp4_quantize.cu", "fp4_matmul.cu", "fp4_matmul_pair.cu", "fp4_experts.cu"]


def binding_path() -> str:
    """Module with the tensor checks of the 8-bit and 4-bit float operators.  It is compiled against the headers of torch and the interpreter, and its
    name says which: after a change of either there is no file to load until it is built again."""
    try:
        torch_version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:  # (not installed as a package)
        import torch

        torch_version = torch.__version__
    tag = "%s-torch-%s" % (sys.implementation.cache_tag, torch_version)
    return os.path.join(HERE, "_binding-%s.so" % "".join(c if c.isalnum() or c in "-." else "_" for c in tag))


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def needs_build(so: str = SO) -> bool:
    if not os.path.exists(so):
        return True
    t = os.path.getmtime(so)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "b2conv.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def binding_command(out: str) -> list:
    import sysconfig

    import torch

    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include"), sysconfig.get_paths()["include"], os.path.join(ROOT, "include")]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI] +
            [x for p in inc for x in ("-I", p)] + ["-o", out, os.path.join(CSRC, "binding.cpp"), "-L", os.path.join(root, "lib"),
                                                   "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"])


def build_binding(force: bool = False) -> str:
    deps = [os.path.join(CSRC, "binding.cpp"), os.path.join(ROOT, "include", "b2conv.h")]
    so = binding_path()
    if not force and os.path.exists(so) and all(os.path.getmtime(d) <= os.path.getmtime(so) for d in deps):
        return so
    tmp = so + ".tmp.%d" % os.getpid()
    subprocess.check_call(binding_command(tmp))
    os.replace(tmp, so)
    return so


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """The library first: it needs nvcc alone.  Then the binding, where there is a torch to bind to."""
    so = build_library(force, verbose, debug)
    if importlib.util.find_spec("torch") is not None:
        build_binding(force and not debug)
    return so


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    so = SO_DEBUG if debug else SO
    if not force and not needs_build(so):
        return so
    cmd = [
        _nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
        "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "-x", "cu", "--threads", "0",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    ]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    if debug:
        cmd += ["-DB2C_DEBUG_BOUNDS"]
    tmp = so + ".tmp.%d" % os.getpid()
    cmd += ["-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, so)
    return so


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
