"""What of the 8-bit float operators can be checked without a device: sources, decisions of the host, refusals."""
import ctypes
import glob
import os
import re
import subprocess

import pytest
import torch

import paper_2104_04731_b200 as b2c

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_04731_b200", "csrc")


def test_results_of_waits_are_voted():
    """The rule of the convolution's kernels (test_bounded_waits): lanes of a warp act on a wait's result together, or some could be at a
    warp-wide instruction, or store a result, without the others."""
    waits = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "fp8_*.cu"))):
        for n, line in enumerate(open(path).read().split("\n")):
            call = re.search(r"\bmbar_wait(_\w+)?\(", line)
            if not call or "__device__" in line or line.lstrip().startswith("//"):
                continue
            waits += 1
            assert line[:call.start()].strip().endswith("__all_sync(0xffffffffu,"), (os.path.basename(path), n + 1, line)
    assert waits >= 10


def test_tensor_memory_goes_back_before_a_cluster_meets():
    """A block of the few-rows kernel that waits for the others of its cluster holds none: with another stream's kernel between them, a
    circle of blocks that hold some and blocks that wait for some would not end."""
    source = open(os.path.join(CSRC, "fp8_matmul.cu")).read()
    kernel = source[source.index("matmul_rows_kernel(const"):]
    assert 0 < kernel.index("tcgen05.alloc") < kernel.index("tcgen05.dealloc") < kernel.index("cluster_sync()")


def test_decisions_about_large_sizes(tmp_path):
    """Sizes that no test can run (results of more than 2 GiB a row): what the host decides about them, as a small program."""
    exe = str(tmp_path / "fp8_decisions")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", os.path.join(cuda, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           os.path.join(ROOT, "tests", "fp8_decisions.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.fixture(scope="module")
def lib():
    from paper_2104_04731_b200 import build

    build.build()
    return b2c.load()


def code_of(call, *args, **kw):
    with pytest.raises(b2c.B2CError) as e:
        call(*args, **kw)
    return e.value.code


@pytest.mark.parametrize("cols", [2 ** 31, 2 ** 32 + 64, 2 ** 33])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_refuses_more_columns_than_its_argument_holds(lib, cols, block):
    """Tensors without memory: the sizes are refused before anything else is asked of them (2^32 + 64 columns were taken as 64)."""
    x = torch.empty(1, cols, dtype=torch.bfloat16, device="meta")
    q = torch.empty(1, cols, dtype=torch.float8_e4m3fn, device="meta")
    assert code_of(b2c.fp8_quantize, x, q, torch.empty(1, -(-cols // 128), device="meta"), block_rows=block) == b2c.E_UNSUPPORTED


@pytest.mark.parametrize("hidden,inter", [(2 ** 31 - 16, 16), (16, 2 ** 31 - 16), (2 ** 30 + 16, 16), (16, 2 ** 30 + 16)])
def test_experts_refuse_what_the_products_refuse(lib, hidden, inter):
    """Columns of a tile past the last one are numbers of 32 bits too; the products take 2^30 columns at most."""
    n = ctypes.c_size_t()
    d = b2c.ExpertsDesc(hidden, inter, 4, 2, b2c.BF16)
    assert lib.b2c_experts_workspace_bytes(ctypes.byref(d), 8, ctypes.byref(n)) == b2c.E_UNSUPPORTED
    p = 1 << 20
    assert lib.b2c_fp8_experts(ctypes.byref(d), 8, p, hidden, p, p, p, p, p, p, p, hidden, p, None) == b2c.E_UNSUPPORTED
    d = b2c.ExpertsDesc(2 ** 30, 16, 4, 2, b2c.BF16)
    assert lib.b2c_experts_workspace_bytes(ctypes.byref(d), 8, ctypes.byref(n)) == b2c.OK


def test_binding_goes_with_its_torch_and_interpreter(lib, monkeypatch):
    """It reads torch's objects, so one that was compiled for another torch or interpreter is neither kept by the build nor loaded."""
    from paper_2104_04731_b200 import build

    here = build.build_binding()
    assert os.path.exists(here) and build.build_binding() == here
    commands = []
    monkeypatch.setattr(build.subprocess, "check_call", commands.append)
    monkeypatch.setattr(build.os, "replace", lambda a, b: None)
    version = build.importlib.metadata.version
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "9.9.9" if name == "torch" else version(name))
    assert build.build_binding() != here and len(commands) == 1
    monkeypatch.setattr(b2c, "_native", None)
    with pytest.raises(ImportError):
        b2c.fp8_quantize(None, None, None)


def test_library_needs_no_torch(monkeypatch):
    """nvcc's part comes first, and is all there is without a torch."""
    from paper_2104_04731_b200 import build

    commands, replaced = [], []
    monkeypatch.setattr(build.subprocess, "check_call", lambda c: commands.append(os.path.basename(c[0])))
    monkeypatch.setattr(build.os, "replace", lambda a, b: replaced.append(b))
    assert build.build(force=True) == build.SO
    assert commands == ["nvcc", "g++"] and replaced[0] == build.SO
    commands.clear()
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    assert build.build(force=True) == build.SO and commands == ["nvcc"]


def test_selftest_refuses_forms_that_are_none(lib):
    assert lib.b2c_selftest_fp8_wait(2, None) == b2c.E_INVALID_ARG
    assert lib.b2c_selftest_fp8_wait(-1, None) == b2c.E_INVALID_ARG
