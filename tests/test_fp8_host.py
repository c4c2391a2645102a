"""Argument checks of the 8-bit float operators: every refusal comes before any CUDA call, so none of this needs a device."""
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


QUANTIZE = dict(x=P, x_type=b2c.BF16, rows=4, cols=256, ldx=256, block=1, q_type=b2c.E4M3, q=P, ldq=256, scale=P, lds=2, stream=None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(q=None), dict(scale=None), dict(x=P + 1), dict(scale=P + 2), dict(x_type=b2c.E4M3), dict(x_type=9),
                                dict(q_type=b2c.BF16), dict(rows=-1), dict(cols=0), dict(ldx=255), dict(ldq=255), dict(lds=1), dict(block=64),
                                dict(block=0)], ids=str)
def test_quantize_refusals(lib, kw):
    assert lib.b2c_fp8_quantize(*with_(QUANTIZE, **kw)) == BAD


def test_quantize_limits(lib):
    assert lib.b2c_fp8_quantize(*with_(QUANTIZE, rows=1 << 31)) == NO
    assert lib.b2c_fp8_quantize(*with_(QUANTIZE, rows=0, x=None, q=None, scale=None)) == b2c.OK


MATMUL = dict(rows=4, a=P, lda=256, a_scale=P, lds=2, b=P, b_scale=P, offsets=None, y=P, ldy=100, stream=None)
DESC = dict(N=100, K=256, groups=1, a_type=b2c.E4M3, b_type=b2c.E5M2, y_type=b2c.F16)


@pytest.mark.parametrize("desc,kw", [(dict(N=0), {}), (dict(K=8), {}), (dict(K=250), {}), (dict(K=0), {}), (dict(groups=0), {}), (dict(groups=2), {}),
                                     (dict(a_type=b2c.F16), {}), (dict(b_type=7), {}), (dict(y_type=b2c.E4M3), {}), ({}, dict(rows=-1)),
                                     ({}, dict(a=None)), ({}, dict(a=P + 8)), ({}, dict(b=None)), ({}, dict(b=P + 4)), ({}, dict(lda=240)),
                                     ({}, dict(lda=264)), ({}, dict(lds=1)), ({}, dict(ldy=99)), ({}, dict(y=P + 1)), ({}, dict(y=None)),
                                     ({}, dict(a_scale=None)), ({}, dict(b_scale=P + 1)), ({}, dict(offsets=P + 2))], ids=str)
def test_matmul_refusals(lib, desc, kw):
    d = b2c.MatmulDesc(*with_(DESC, **desc))
    assert lib.b2c_fp8_matmul(ctypes.byref(d), *with_(MATMUL, **kw)) == BAD


def test_matmul_limits(lib):
    d = b2c.MatmulDesc(*with_(DESC, groups=1025))
    assert lib.b2c_fp8_matmul(ctypes.byref(d), *with_(MATMUL, offsets=P)) == NO
    d = b2c.MatmulDesc(*with_(DESC))
    assert lib.b2c_fp8_matmul(ctypes.byref(d), *with_(MATMUL, rows=1 << 31)) == NO
    assert lib.b2c_fp8_matmul(ctypes.byref(d), *with_(MATMUL, lda=1 << 40)) == NO
    wide = b2c.MatmulDesc(*with_(DESC, N=1 << 22, K=1 << 20))
    assert lib.b2c_fp8_matmul(ctypes.byref(wide), *with_(MATMUL, lda=1 << 20, lds=1 << 13, ldy=1 << 22)) == NO
    assert lib.b2c_fp8_matmul(ctypes.byref(d), *with_(MATMUL, rows=0, a=None)) == b2c.OK
    assert lib.b2c_fp8_matmul(None, *with_(MATMUL)) == BAD


ROUTE = dict(experts=64, topk=4, score=0, groups=4, topk_groups=2, group_score=1, renormalise=1, logit_type=b2c.F32, scale=1.0)
ROUTE_ARGS = dict(tokens=3, logits=P, ld=64, bias=None, weights=P, ids=P, stream=None)


@pytest.mark.parametrize("desc,kw", [(dict(experts=0), {}), (dict(topk=0), {}), (dict(topk=33, groups=1, topk_groups=1, experts=32), {}), (dict(topk=17, topk_groups=1), {}),
                                     (dict(groups=5), {}), (dict(groups=0), {}), (dict(topk_groups=5), {}), (dict(topk_groups=0), {}),
                                     (dict(score=2), {}), (dict(group_score=-1), {}), (dict(renormalise=2), {}), (dict(logit_type=b2c.E4M3), {}),
                                     ({}, dict(tokens=-1)), ({}, dict(ld=63)), ({}, dict(logits=None)), ({}, dict(logits=P + 2)), ({}, dict(bias=P + 1)),
                                     ({}, dict(weights=None)), ({}, dict(ids=P + 2))], ids=str)
def test_route_refusals(lib, desc, kw):
    d = b2c.RouteDesc(*with_(ROUTE, **desc))
    assert lib.b2c_route(ctypes.byref(d), *with_(ROUTE_ARGS, **kw)) == BAD


def test_route_limits(lib):
    for kw in (dict(experts=1028), dict(topk=33, groups=1, topk_groups=1), dict(experts=128, groups=64, topk_groups=64)):
        d = b2c.RouteDesc(*with_(ROUTE, **kw))
        assert lib.b2c_route(ctypes.byref(d), *with_(ROUTE_ARGS, ld=2000)) == NO, kw
    assert lib.b2c_route(ctypes.byref(b2c.RouteDesc(*with_(ROUTE))), *with_(ROUTE_ARGS, tokens=0, logits=None)) == b2c.OK


def test_sort_and_combine_refusals(lib):
    n = ctypes.c_size_t(99)
    assert lib.b2c_route_sort_workspace_bytes(-1, 4, ctypes.byref(n)) == BAD
    assert lib.b2c_route_sort_workspace_bytes(4, 0, ctypes.byref(n)) == BAD
    assert lib.b2c_route_sort_workspace_bytes(4, 4, None) == BAD
    assert lib.b2c_route_sort_workspace_bytes(4, 1025, ctypes.byref(n)) == NO
    assert lib.b2c_route_sort_workspace_bytes(16, 4, ctypes.byref(n)) == b2c.OK and n.value == 0
    sort = dict(ids=P, pairs=5000, experts=8, offsets=P, rows=P, order=None, ws=P, stream=None)
    for kw in (dict(ids=None), dict(pairs=-1), dict(experts=0), dict(offsets=None), dict(rows=None), dict(order=P + 1), dict(ws=None), dict(ws=P + 8), dict(ids=P + 1)):
        assert lib.b2c_route_sort(*with_(sort, **kw)) == BAD, kw
    combine = dict(y=P, y_type=b2c.BF16, y_rows=10, ldy=64, rows=P, weights=P, tokens=3, topk=2, cols=64, out=P, out_type=b2c.BF16, ldo=64, stream=None)
    for kw in (dict(y=None), dict(y_type=b2c.E4M3), dict(y_rows=-1), dict(ldy=63), dict(rows=None), dict(weights=None), dict(tokens=-1), dict(topk=0),
               dict(cols=0), dict(out=None), dict(out=P + 1), dict(out_type=5), dict(ldo=63), dict(rows=P + 1)):
        assert lib.b2c_route_combine(*with_(combine, **kw)) == BAD, kw
    assert lib.b2c_route_combine(*with_(combine, topk=33)) == NO
    assert lib.b2c_route_combine(*with_(combine, tokens=0)) == b2c.OK


EXPERTS = dict(hidden=256, inter=128, experts=8, topk=2, type=b2c.BF16)
EXPERTS_ARGS = dict(tokens=3, x=P, ldx=256, ids=P, weights=P, w1=P, s1=P, w2=P, s2=P, y=P, ldy=256, ws=P, stream=None)


@pytest.mark.parametrize("desc,kw", [(dict(hidden=250), {}), (dict(hidden=0), {}), (dict(inter=8), {}), (dict(experts=0), {}), (dict(topk=0), {}), (dict(topk=9), {}),
                                     (dict(type=b2c.E4M3), {})] + [({}, {k: None}) for k in ("x", "ids", "weights", "w1", "s1", "w2", "s2", "y", "ws")] +
                         [({}, dict(tokens=-1)), ({}, dict(ldx=255)), ({}, dict(ldy=100)), ({}, dict(w1=P + 8)), ({}, dict(w2=P + 1)), ({}, dict(ws=P + 4)),
                          ({}, dict(x=P + 1))], ids=str)
def test_experts_refusals(lib, desc, kw):
    d = b2c.ExpertsDesc(*with_(EXPERTS, **desc))
    assert lib.b2c_fp8_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, **kw)) == BAD


def test_experts_limits_and_workspace(lib):
    n = ctypes.c_size_t()
    assert lib.b2c_fp8_experts(None, *with_(EXPERTS_ARGS)) == BAD
    d = b2c.ExpertsDesc(*with_(EXPERTS, experts=1025))
    assert lib.b2c_fp8_experts(ctypes.byref(d), *with_(EXPERTS_ARGS)) == NO
    d = b2c.ExpertsDesc(*with_(EXPERTS))
    assert lib.b2c_fp8_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, tokens=1 << 31)) == NO
    assert lib.b2c_fp8_experts(ctypes.byref(d), *with_(EXPERTS_ARGS, tokens=0, x=None)) == b2c.OK
    assert lib.b2c_experts_workspace_bytes(ctypes.byref(d), 3, None) == BAD
    sizes = []
    for tokens in (0, 1, 100, 100000):
        assert lib.b2c_experts_workspace_bytes(ctypes.byref(d), tokens, ctypes.byref(n)) == b2c.OK
        sizes.append(n.value)
        # rows in 8 bits and their scales, twice, and the rows of the result
        assert n.value >= tokens * 2 * (256 + 8 + 128 + 4 + 2 * 256)
    assert sizes == sorted(sizes)
    assert lib.b2c_fp8_status(None) == BAD


def refused(call, *args, code=BAD, **kw):
    with pytest.raises(b2c.B2CError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_binding_refuses_what_the_library_cannot_see(lib):
    """Shapes, strides, types and devices of tensors; nothing of this reaches the library."""
    f8 = torch.float8_e4m3fn
    x, q, s = torch.zeros(4, 256), torch.zeros(4, 256).to(f8), torch.zeros(4, 2)
    refused(b2c.fp8_quantize, x, q[:3], s)
    refused(b2c.fp8_quantize, x, q, s[:, :1])
    refused(b2c.fp8_quantize, x, q, s, block_rows=128)
    refused(b2c.fp8_quantize, x, q, s, block_rows=2)
    refused(b2c.fp8_quantize, x, q, s.double())
    refused(b2c.fp8_quantize, x, q, s)  # not on the device
    refused(b2c.fp8_quantize, x, q, None)
    refused(b2c.fp8_quantize, x.t()[:4, :4], q[:, :4], s[:, :1])
    refused(b2c.fp8_quantize, x[:1].expand(4, 256), q, s)
    a, sa, b, sb, y = q, s, torch.zeros(100, 256).to(f8), torch.zeros(1, 2), torch.zeros(4, 100)
    for args in [(a[:, :128], sa, b, sb, y), (a, sa[:, :1], b, sb, y), (a, sa, b, sb[:, :1], y), (a, sa, b, sb, y[:, :99]), (a, sa, b.t(), sb, y),
                 (a, sa.double(), b, sb, y), (a, sa, b[None], sb[None], y), (a, sa, b, sb, y)]:
        refused(b2c.fp8_matmul, *args)
    refused(b2c.fp8_matmul, a, sa, b, sb, y, offsets=torch.zeros(2, dtype=torch.int32))
    refused(b2c.fp8_matmul, a, sa, b[None], sb[None], y, offsets=torch.zeros(2, dtype=torch.int64))
    refused(b2c.fp8_matmul, a, sa, b[None], sb[None], y, offsets=torch.zeros(3, dtype=torch.int32))
    d = b2c.make_route_desc(8, 2)
    w, i = torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32)
    for args in [(torch.zeros(4, 9), w, i), (torch.zeros(4, 8), w[:, :1], i), (torch.zeros(4, 8), w, i.long()), (torch.zeros(4, 8), w.double(), i), (torch.zeros(4, 8), w, i)]:
        refused(b2c.route, d, *args)
    refused(b2c.route, d, torch.zeros(4, 8), w, i, bias=torch.zeros(7))
    refused(b2c.route_sort, i, 8, torch.zeros(8, dtype=torch.int32), i.clone())
    refused(b2c.route_sort, i.long(), 8, torch.zeros(9, dtype=torch.int32), i.clone())
    refused(b2c.route_sort, torch.zeros(5000, dtype=torch.int32), 8, torch.zeros(9, dtype=torch.int32), torch.zeros(5000, dtype=torch.int32),
            code=b2c.E_WORKSPACE_TOO_SMALL)
    refused(b2c.route_combine, torch.zeros(8, 16), i, w, torch.zeros(4, 15))
    refused(b2c.route_combine, torch.zeros(8, 16), i, w.t(), torch.zeros(4, 16))
    h = torch.zeros(4, 128)
    w1, s1, w2, s2 = torch.zeros(8, 2, 16, 128).to(f8), torch.zeros(8, 2, 1, 1), torch.zeros(8, 128, 16).to(f8), torch.zeros(8, 1, 1)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for args in [(h[:, :64], i, w, w1, s1, w2, s2, h, ws), (h, i[:3], w, w1, s1, w2, s2, h, ws), (h, i, w, w1[:, :1], s1, w2, s2, h, ws),
                 (h, i, w, w1, s1, w2.transpose(1, 2), s2, h, ws), (h, i, w, w1.float(), s1, w2, s2, h, ws), (h, i, w, w1, s1[:7], w2, s2, h, ws),
                 (h, i, w, w1, s1, w2, s2, h.half(), ws), (h, i, w, w1, s1, w2, s2, h, ws)]:
        refused(b2c.fp8_experts, *args)
