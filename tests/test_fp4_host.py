"""Argument checks of the 4-bit float operators: every refusal comes before any CUDA call, so none of this needs a device."""
import ctypes

import pytest
import torch

import paper_2104_04731_b200 as b2c

P = 1 << 20  # a well aligned address that no refused call may touch
BAD, NO = b2c.E_INVALID_ARG, b2c.E_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    from paper_2104_04731_b200 import build

    build.build()
    return b2c.load()


def with_(base, **kw):
    assert set(kw) <= set(base)
    return list({**base, **kw}.values())


QUANTIZE = dict(x=P, x_type=b2c.BF16, rows=4, cols=255, ldx=256, format=b2c.NVFP4, factor=P, q=P, ldq=128, scale=P, lds=16, stream=None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(q=None), dict(scale=None), dict(x=P + 1), dict(factor=P + 2), dict(x_type=b2c.E4M3), dict(x_type=9), dict(format=2),
                                dict(format=-1), dict(format=b2c.MXFP4), dict(rows=-1), dict(cols=0), dict(ldx=254), dict(ldq=127), dict(lds=15)], ids=str)
def test_quantize_refusals(lib, kw):
    assert lib.b2c_fp4_quantize(*with_(QUANTIZE, **kw)) == BAD


DEQUANTIZE = dict(q=P, ldq=128, scale=P, lds=16, rows=4, cols=255, format=b2c.NVFP4, factor=P, y=P, y_type=b2c.BF16, ldy=256, stream=None)


@pytest.mark.parametrize("kw", [dict(y=None), dict(q=None), dict(scale=None), dict(y=P + 1), dict(factor=P + 2), dict(y_type=b2c.E4M3), dict(format=2),
                                dict(format=b2c.MXFP4), dict(rows=-1), dict(cols=0), dict(ldy=254), dict(ldq=127), dict(lds=15)], ids=str)
def test_dequantize_refusals(lib, kw):
    assert lib.b2c_fp4_dequantize(*with_(DEQUANTIZE, **kw)) == BAD


def test_quantize_limits(lib):
    for call, base in ((lib.b2c_fp4_quantize, QUANTIZE), (lib.b2c_fp4_dequantize, DEQUANTIZE)):
        assert call(*with_(base, rows=1 << 31)) == NO
        big = (1 << 30) + 1
        assert call(*with_(base, cols=big, **{k: 1 << 31 for k in base if k.startswith("ld")})) == NO
        assert call(*with_(base, rows=0, q=None, scale=None)) == b2c.OK


MATMUL = dict(rows=4, a=P, lda=128, a_scale=P, lda_s=16, b=P, b_scale=P, ldb_s=16, alpha=None, offsets=None, y=P, ldy=100, stream=None)
DESC = dict(N=100, K=256, groups=1, format=b2c.NVFP4, y_type=b2c.F16)


@pytest.mark.parametrize("desc,kw", [(dict(N=0), {}), (dict(K=16), {}), (dict(K=240), {}), (dict(K=0), {}), (dict(groups=0), {}), (dict(groups=2), {}), (dict(format=2), {}),
                                     (dict(y_type=b2c.E4M3), {}), ({}, dict(rows=-1)), ({}, dict(a=None)), ({}, dict(a=P + 8)), ({}, dict(b=None)), ({}, dict(b=P + 4)),
                                     ({}, dict(lda=112)), ({}, dict(lda=136)), ({}, dict(lda_s=8)), ({}, dict(lda_s=24)), ({}, dict(ldb_s=0)), ({}, dict(ldb_s=17)),
                                     (dict(K=512), dict(lda=256, ldb_s=32)), ({}, dict(ldy=99)), ({}, dict(y=P + 1)), ({}, dict(y=None)), ({}, dict(a_scale=None)),
                                     ({}, dict(a_scale=P + 8)), ({}, dict(b_scale=P + 1)), ({}, dict(alpha=P + 2)), ({}, dict(offsets=P + 2))], ids=str)
def test_matmul_refusals(lib, desc, kw):
    d = b2c.Fp4MatmulDesc(*with_(DESC, **desc))
    assert lib.b2c_fp4_matmul(ctypes.byref(d), *with_(MATMUL, **kw)) == BAD


def test_matmul_limits(lib):
    d = b2c.Fp4MatmulDesc(*with_(DESC, groups=1025))
    assert lib.b2c_fp4_matmul(ctypes.byref(d), *with_(MATMUL, offsets=P)) == NO
    d = b2c.Fp4MatmulDesc(*with_(DESC))
    for kw in (dict(rows=1 << 31), dict(lda=1 << 40), dict(lda_s=1 << 40), dict(ldb_s=1 << 40), dict(ldy=1 << 40)):
        assert lib.b2c_fp4_matmul(ctypes.byref(d), *with_(MATMUL, **kw)) == NO, kw
    wide = b2c.Fp4MatmulDesc(*with_(DESC, N=1 << 22, K=1 << 20))
    assert lib.b2c_fp4_matmul(ctypes.byref(wide), *with_(MATMUL, lda=1 << 19, lda_s=1 << 16, ldb_s=1 << 16, ldy=1 << 22)) == NO
    assert lib.b2c_fp4_matmul(ctypes.byref(d), *with_(MATMUL, rows=0, a=None)) == b2c.OK
    assert lib.b2c_fp4_matmul(None, *with_(MATMUL)) == BAD


EXPERTS = dict(hidden=256, inter=128, experts=8, topk=2, type=b2c.BF16, format=b2c.NVFP4)
EXPERTS_ARGS = dict(tokens=3, x=P, ldx=256, ids=P, weights=P, w1=P, s1=P, ld1=16, w2=P, s2=P, ld2=16, gx=None, g1=None, gh=None, g2=None, y=P, ldy=256, ws=P, stream=None)


@pytest.mark.parametrize("desc,kw", [(dict(hidden=240), {}), (dict(hidden=0), {}), (dict(inter=16), {}), (dict(inter=144), {}), (dict(experts=0), {}), (dict(topk=0), {}),
                                     (dict(topk=9), {}), (dict(type=b2c.E4M3), {}), (dict(format=3), {})] +
                         [({}, {k: None}) for k in ("x", "ids", "weights", "w1", "s1", "w2", "s2", "y", "ws")] +
                         [({}, dict(tokens=-1)), ({}, dict(ldx=255)), ({}, dict(ldy=100)), ({}, dict(w1=P + 8)), ({}, dict(w2=P + 1)), ({}, dict(ws=P + 4)), ({}, dict(s1=P + 8)),
                          ({}, dict(s2=P + 4)), ({}, dict(ld1=8)), ({}, dict(ld2=20)), ({}, dict(ld1=24)), ({}, dict(x=P + 1)), ({}, dict(gx=P + 1)), ({}, dict(g2=P + 2))] +
                         [(dict(format=b2c.MXFP4), {k: P}) for k in ("gx", "g1", "gh", "g2")], ids=str)
def test_experts_refusals(lib, desc, kw):
    d = b2c.Fp4ExpertsDesc(*with_(EXPERTS, **desc))
    assert lib.b2c_fp4_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, **kw)) == BAD


def test_experts_limits_and_workspace(lib):
    n = ctypes.c_size_t()
    assert lib.b2c_fp4_experts(None, *with_(EXPERTS_ARGS)) == BAD
    d = b2c.Fp4ExpertsDesc(*with_(EXPERTS, experts=1025))
    assert lib.b2c_fp4_experts(ctypes.byref(d), *with_(EXPERTS_ARGS)) == NO
    d = b2c.Fp4ExpertsDesc(*with_(EXPERTS))
    assert lib.b2c_fp4_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, tokens=1 << 31)) == NO
    assert lib.b2c_fp4_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, ld1=1 << 36)) == NO
    assert lib.b2c_fp4_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, tokens=0, x=None)) == b2c.OK
    assert lib.b2c_fp4_experts_workspace_bytes(ctypes.byref(d), 3, None) == BAD
    sizes = []
    for tokens in (0, 1, 100, 100000):
        assert lib.b2c_fp4_experts_workspace_bytes(ctypes.byref(d), tokens, ctypes.byref(n)) == b2c.OK
        sizes.append(n.value)
        # rows in 4 bits and their scales, twice, and the rows of the result
        assert n.value >= tokens * 2 * (128 + 16 + 64 + 16 + 4 * 256)
    assert sizes == sorted(sizes)
    assert lib.b2c_fp4_status(None) == BAD
    assert lib.b2c_selftest_fp4_wait(3, None) == BAD


def refused(call, *args, code=BAD, **kw):
    with pytest.raises(b2c.B2CError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_room_for_scales():
    for fmt, cols, pitch in ((b2c.MXFP4, 32, 16), (b2c.MXFP4, 512, 16), (b2c.MXFP4, 513, 32), (b2c.NVFP4, 256, 16), (b2c.NVFP4, 257, 32), (b2c.NVFP4, 1, 16)):
        assert b2c.fp4_scale_pitch(cols, fmt) == pitch
        q, s = b2c.fp4_empty((2, 3), cols, fmt, device="cpu")
        assert q.shape == (2, 3, (cols + 1) // 2) and s.shape == (2, 3, -(-cols // (32 if fmt == b2c.MXFP4 else 16)))
        assert s.stride(1) == pitch and s.stride(0) == 3 * pitch


def test_binding_refuses_what_the_library_cannot_see(lib):
    """Shapes, strides, types and devices of tensors; nothing of this reaches the library."""
    x = torch.zeros(4, 256)
    q, s = b2c.fp4_empty(4, 256, b2c.NVFP4, device="cpu")
    mx_q, mx_s = b2c.fp4_empty(4, 256, b2c.MXFP4, device="cpu")
    g = torch.ones(1)
    refused(b2c.fp4_quantize, x, q[:3], s)
    refused(b2c.fp4_quantize, x, q, s[:, :1])
    refused(b2c.fp4_quantize, x, q, mx_s[:3])
    refused(b2c.fp4_quantize, x, q.int(), s)
    refused(b2c.fp4_quantize, x, q, s.view(torch.uint8))
    refused(b2c.fp4_quantize, x.double(), q, s)
    refused(b2c.fp4_quantize, x, q, s, global_scale=torch.ones(2))
    refused(b2c.fp4_quantize, x, q, s, global_scale=g.double())
    refused(b2c.fp4_quantize, x.t().contiguous().t(), q, s)
    refused(b2c.fp4_quantize, x[:1].expand(4, 256), q, s)
    refused(b2c.fp4_quantize, x, q, s)  # (not on a device)
    refused(b2c.fp4_quantize, "x", q, s)
    refused(b2c.fp4_dequantize, q, s, x[:, :250])
    refused(b2c.fp4_dequantize, q, s[:, 1:], x)
    refused(b2c.fp4_dequantize, q, s, x.int())
    refused(b2c.fp4_dequantize, q, s, x)
    b, bs = b2c.fp4_empty(8, 256, b2c.NVFP4, device="cpu")
    y = torch.zeros(4, 8)
    refused(b2c.fp4_matmul, q, s, b, bs, y[:, :7])
    refused(b2c.fp4_matmul, q, s, b[:, :100], bs, y)
    refused(b2c.fp4_matmul, q, mx_s, b, bs, y)
    refused(b2c.fp4_matmul, q, s, b[None], bs[None], y)
    refused(b2c.fp4_matmul, q, s, b, bs, y, offsets=torch.zeros(2, dtype=torch.int32))
    refused(b2c.fp4_matmul, q, s, b, bs, y, alpha=torch.ones(3))
    stack, stack_s = b2c.fp4_empty((2, 8), 256, b2c.NVFP4, device="cpu")
    off = torch.zeros(3, dtype=torch.int32)
    refused(b2c.fp4_matmul, q, s, stack, stack_s, y, alpha=g, offsets=off)
    refused(b2c.fp4_matmul, q, s, stack, stack_s, y, offsets=off.long())
    refused(b2c.fp4_matmul, q, s, stack, stack_s[:, ::2].repeat_interleave(2, 1)[:, :8].transpose(0, 1).contiguous().transpose(0, 1), y, offsets=off)
    refused(b2c.fp4_matmul, q, s, stack, stack_s, y, offsets=off)
    w1, s1 = b2c.fp4_empty((2, 2, 64), 256, b2c.NVFP4, device="cpu")
    w2, s2 = b2c.fp4_empty((2, 256), 64, b2c.NVFP4, device="cpu")
    ids, w, out, ws = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4, 256), torch.zeros(1 << 20, dtype=torch.uint8)
    fine = dict(x=x, ids=ids, weights=w, w1=w1, w1_scale=s1, w2=w2, w2_scale=s2, y=out, workspace=ws)
    for kw in (dict(ids=ids.long()), dict(weights=w[:, :1]), dict(w1=w1[:, :1]), dict(w1_scale=s1[..., :3]), dict(w2=w2[:1]), dict(w2_scale=mx_s), dict(y=out[:3]),
               dict(y=out.half()), dict(x_global=torch.ones(2)), dict(w1_global=torch.ones(1)), dict(h_global=torch.ones(2)), dict(w2_global=torch.ones(3)), dict()):
        refused(b2c.fp4_experts, **{**fine, **kw})
