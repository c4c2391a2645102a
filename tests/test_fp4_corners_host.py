"""What of the 4-bit float operators can be checked without a device: refusals of unusual tensors, decisions of the host."""
import os
import subprocess

import pytest
import torch

import paper_2104_04731_b200 as b2c

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_04731_b200", "csrc")


def test_decisions_about_large_groups(tmp_path):
    """Sizes that no test can run (a group of more than 1.4e9 rows), as a small program."""
    exe = str(tmp_path / "fp4_decisions")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", os.path.join(cuda, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           os.path.join(ROOT, "tests", "fp4_decisions.cpp"), "-o", exe])
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


def layer(hidden, inter, experts=2, tokens=4, topk=2, fmt=b2c.NVFP4):
    """Arguments of an expert layer, on the CPU."""
    (w1, s1), (w2, s2) = (b2c.fp4_empty(shape, cols, fmt, device="cpu") for shape, cols in (((experts, 2, inter), hidden), ((experts, hidden), inter)))
    return dict(x=torch.zeros(tokens, hidden), ids=torch.zeros(tokens, topk, dtype=torch.int32), weights=torch.zeros(tokens, topk), w1=w1, w1_scale=s1, w2=w2,
                w2_scale=s2, y=torch.zeros(tokens, hidden), workspace=torch.zeros(1 << 20, dtype=torch.uint8))


@pytest.mark.parametrize("fmt", [b2c.MXFP4, b2c.NVFP4], ids=["mx", "nv"])
@pytest.mark.parametrize("groups,N,K", [(4, 0, 64), (1, 0, 64), (0, 8, 64), (4, 8, 0), (4, 0, 0)])
def test_product_refuses_empty_stacks(lib, groups, N, K, fmt):
    """Matrices without rows or columns, or none at all: the distance between rows was sought by a remainder by 0, which ended the process."""
    q, s = b2c.fp4_empty(3, K, fmt, device="cpu")
    b, bs = b2c.fp4_empty((groups, N), K, fmt, device="cpu")
    assert code_of(b2c.fp4_matmul, q, s, b, bs, torch.zeros(3, N), offsets=torch.zeros(groups + 1, dtype=torch.int32)) == b2c.E_INVALID_ARG


@pytest.mark.parametrize("fmt", [b2c.MXFP4, b2c.NVFP4], ids=["mx", "nv"])
@pytest.mark.parametrize("kw", [dict(hidden=256, inter=0), dict(hidden=0, inter=64), dict(hidden=0, inter=0), dict(hidden=256, inter=64, experts=0)], ids=str)
def test_experts_refuse_empty_matrices(lib, kw, fmt):
    assert code_of(b2c.fp4_experts, **layer(fmt=fmt, **kw)) == b2c.E_INVALID_ARG


@pytest.mark.parametrize("shape", [(), (4,), (1024,), (4, 256, 1), (1, 4, 256)], ids=str)
def test_experts_refuse_results_that_are_no_matrix(lib, shape):
    """As every refusal by an error of the library, in 8 bits and in 4 (torch's own came out for a y of fewer dimensions)."""
    args = layer(256, 64)
    assert code_of(b2c.fp4_experts, **{**args, "y": torch.zeros(shape)}) == b2c.E_INVALID_ARG
    w1, w2 = torch.zeros(2, 2, 64, 256).to(torch.float8_e4m3fn), torch.zeros(2, 256, 64).to(torch.float8_e4m3fn)
    eight = dict(args, w1=w1, w1_scale=torch.zeros(2, 2, 1, 2), w2=w2, w2_scale=torch.zeros(2, 2, 1), y=torch.zeros(shape))
    assert code_of(b2c.fp8_experts, **eight) == b2c.E_INVALID_ARG
