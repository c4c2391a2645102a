"""4-bit float operators on the device against their definitions in 64 bits (fp4_ref)."""
import math

import pytest
import torch

import fp4_ref as ref
from fp4_ref import MX, NV

pytestmark = pytest.mark.gpu

WIDE = [torch.float32, torch.float16, torch.bfloat16]
FMT = pytest.mark.parametrize("fmt", [MX, NV], ids=["mx", "nv"])


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def room(rows, cols, fmt, ldq=None, lds=None):
    """(whole q, q, whole scale, scale): outputs in wider rows, filled with a pattern."""
    wq = torch.full((rows, ldq or (cols + 1) // 2), 0xA5, dtype=torch.uint8, device="cuda")
    ws = torch.full((rows, lds or ref.nb(cols, fmt)), 0x5A, dtype=torch.uint8, device="cuda")
    return wq, wq[:, :(cols + 1) // 2], ws, ws[:, :ref.nb(cols, fmt)].view(ref.SCALE[fmt])


def run_quantize(lib, x, fmt, g=None, ldq=None, lds=None):
    rows, cols = x.shape
    wq, q, ws, s = room(rows, cols, fmt, ldq, lds)
    lib.fp4_quantize(x, q, s, global_scale=g)
    torch.cuda.synchronize()
    assert bool((wq[:, (cols + 1) // 2:] == 0xA5).all()) and bool((ws[:, ref.nb(cols, fmt):] == 0x5A).all())
    if cols % 2:
        assert bool((q[:, -1] >> 4 == 0).all())
    return q, s


def check_quantize(x, fmt, q, s, g=None):
    """Equal in every value: the operator's results are those of the real quotients."""
    want, scale = ref.quantize(x, fmt, g)
    got = ref.scale_numbers(s, fmt)
    assert bool((got.isnan() == scale.isnan()).all())
    assert bool((torch.where(got.isnan(), 0.0, got) == torch.where(scale.isnan(), 0.0, scale)).all())
    assert bool((ref.unpack(q, x.shape[1]) == want).all())


def factor(v):
    return torch.tensor([v], dtype=torch.float32, device="cuda")


# ---- quantisation ----------------------------------------------------------------------------------------------------------------

@FMT
@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 1), (3, 127), (5, 129), (64, 384), (130, 1000), (257, 128), (1, 8192), (7, 15), (40, 48)])
def test_quantize(lib, rows, cols, xt, fmt):
    x = (torch.randn(rows, cols, generator=gen(rows + cols), device="cuda") * 3).to(xt)
    q, s = run_quantize(lib, x, fmt)
    check_quantize(x, fmt, q, s)


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("g", [1.0, 0.0123, 3.7e-4, 2.0 ** -9, 1.25, 2.0 ** -90, 7.7e25, 1.0000001])
@pytest.mark.parametrize("cols", [512, 333])
def test_quantize_factor(lib, cols, g, xt):
    """Factors of few bits (the quotient is formed exactly) and of many; blocks beyond the largest scale, and below the least."""
    x = torch.randn(200, cols, generator=gen(1), device="cuda") * 3
    f = factor(g)
    x[::5] *= 100 * g
    x[1::5] *= 5000 * g
    x[2::5] *= 2.0 ** -8 * g
    x = x.clamp(-1e30, 1e30).to(xt)
    if xt == torch.float16:
        x = x.clamp(-6e4, 6e4)
    q, s = run_quantize(lib, x, NV, f)
    check_quantize(x, NV, q, s, f)


@FMT
def test_quantize_ties(lib, fmt):
    """Half way between two values, and one unit of fp32 beside it, for every border, both signs, and scales of all mantissas."""
    v = torch.tensor(ref.VALUES, dtype=torch.float64)
    mid = (v[:-1] + v[1:]) / 2
    for step in [1.0, 2.0 ** -20, 2.0 ** 40] + ([] if fmt == MX else [1.125, 1.875, 1.375 * 2.0 ** -6, 3 * 2.0 ** -9]):
        t = (torch.cat([mid, -mid]) * step).float()
        x = torch.cat([t, t.nextafter(torch.tensor(math.inf)), t.nextafter(torch.tensor(-math.inf))])
        x = torch.nn.functional.pad(x, (0, -x.numel() % 15)).reshape(-1, 15)
        x = torch.nn.functional.pad(x, (0, ref.BLOCK[fmt] - 15))
        x[:, 15] = 6 * step  # the block's scale is the step
        if fmt == MX or 2.0 ** -9 <= step <= 448:
            x = x.cuda()
            q, s = run_quantize(lib, x, fmt)
            assert bool((ref.scale_numbers(s, fmt) == step).all())
            check_quantize(x, fmt, q, s)


@pytest.mark.parametrize("g", [1.0, 0.37, 0.3333333])
def test_quantize_ties_of_scales(lib, g):
    """amax half way between two E4M3 scales, and one unit beside it."""
    codes = torch.arange(0, 126, dtype=torch.uint8)
    t = ref.scale_numbers(codes.view(torch.float8_e4m3fn), NV)
    f = factor(g)
    a = ((t[:-1] + t[1:]) / 2 * 6 * float(f)).float()
    x = torch.zeros(3, a.numel(), 16)
    x[0, :, 3], x[1, :, 7], x[2, :, 11] = a, -a.nextafter(torch.tensor(math.inf)), a.nextafter(torch.tensor(0.0))
    x = x.reshape(3, -1).cuda()
    q, s = run_quantize(lib, x, NV, f)
    check_quantize(x, NV, q, s, f)


@pytest.mark.parametrize("g", [0.77, 0.0123])
def test_quantize_next_to_borders(lib, g):
    """fp32 numbers within a few units of the borders under a factor of 24 bits."""
    f = factor(g)
    v = torch.tensor(ref.VALUES, dtype=torch.float64)
    mid = (v[:-1] + v[1:]) / 2
    rows = []
    for code in range(40, 120, 3):
        s = float(ref.scale_numbers(torch.tensor([code], dtype=torch.uint8).view(torch.float8_e4m3fn), NV))
        base = (mid * s * float(f)).float()
        for d in range(-5, 6):
            near = (base.view(torch.int32) + d).view(torch.float32)
            rows.append(torch.cat([near, -near, torch.tensor([6 * s * float(f), 0.0])]))
    x = torch.stack(rows).cuda()
    q, s = run_quantize(lib, x, NV, f)
    check_quantize(x, NV, q, s, f)


@FMT
@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("rows,cols,first", [(300, 777, 0), (300, 640, 3), (4000, 2048, 0)])
def test_quantize_special_values(lib, rows, cols, first, xt, fmt):
    """Rows off the 16-byte grid and very many blocks: NaN, infinities, zeros of both signs, the smallest and the largest values."""
    x = torch.randn(rows, first + cols, generator=gen(4), device="cuda").to(xt)[:, first:]
    tiny, large = torch.finfo(xt).tiny, torch.finfo(xt).max
    spots = torch.rand(rows, cols, generator=gen(5), device="cuda")
    x[1::64][spots[1::64] < 2e-3] = math.nan
    x[100::128][spots[100::128] < 2e-3] = math.inf
    x[101::128][spots[101::128] < 1e-3] = -math.inf
    x[130::256] = -0.0
    x[131::256] = tiny / 4
    x[132::256][spots[132::256] < 0.01] = -large
    x[133::256] = tiny * 1.5
    x[2] = 0.0
    q, s = run_quantize(lib, x, fmt)
    check_quantize(x, fmt, q, s)


@FMT
def test_quantize_strides_and_alignment(lib, fmt):
    base = torch.randn(70, 1024, generator=gen(4), device="cuda").bfloat16()
    for x, ldq, lds in [(base[:, 3:500], 511, 33), (base[::2, 8:520], 264, None), (base[:, :512], 257, 40), (base[:1, 1:130], None, None), (base[:, :512], 260, 64)]:
        q, s = run_quantize(lib, x, fmt, None, ldq, lds)
        check_quantize(x, fmt, q, s)


def test_quantize_no_rows(lib):
    q, s = lib.fp4_empty(0, 64, lib.MXFP4)
    lib.fp4_quantize(torch.zeros(0, 64, device="cuda"), q, s)
    lib.fp4_dequantize(q, s, torch.zeros(0, 64, device="cuda"))


def test_packed_type(lib):
    """torch's own packed type in the place of bytes."""
    x = torch.randn(4, 64, generator=gen(2), device="cuda")
    q, s = lib.fp4_empty(4, 64, lib.NVFP4)
    lib.fp4_quantize(x, q.view(torch.float4_e2m1fn_x2), s)
    check_quantize(x, NV, q, s)


# ---- and back --------------------------------------------------------------------------------------------------------------------

@FMT
@pytest.mark.parametrize("yt", WIDE, ids=str)
@pytest.mark.parametrize("rows,cols,ldy", [(1, 32, None), (1, 1, None), (3, 127, 130), (64, 384, None), (33, 1001, None), (257, 136, 144), (2, 8192, None), (9, 40, 41)])
def test_dequantize(lib, rows, cols, ldy, yt, fmt):
    """All codes; scales of all sizes (fp32 holds every product, one rounding to the type; with a factor one more)."""
    g = gen(rows + cols)
    q = torch.randint(0, 256, (rows, (cols + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.randint(0, 255 if fmt == MX else 127, (rows, ref.nb(cols, fmt)), generator=g, device="cuda", dtype=torch.uint8)
    s[0, -1] = 255 if fmt == MX else 127  # NaN
    for f in [None] + ([factor(0.0371)] if fmt == NV else []):
        whole = torch.full((rows, ldy or cols), 7.0, device="cuda", dtype=yt)
        y = whole[:, :cols]
        lib.fp4_dequantize(q, s.view(ref.SCALE[fmt]), y, global_scale=f)
        want = ref.values(q, s, fmt, cols)
        assert bool((whole[:, cols:] == 7.0).all())
        if f is not None:
            want = (want * f.double()).float().double()  # rounded to fp32 first
        else:
            want = torch.where(want.abs() >= 2.0 ** 128, torch.copysign(torch.full_like(want, math.inf), want), want)  # (a NaN stays)
        assert bool((y.isnan() == want.isnan()).all())
        assert bool((torch.nan_to_num(y.double()) == torch.nan_to_num(want.float().to(yt).double())).all())


@FMT
def test_there_and_back(lib, fmt):
    """What 4 bits hold is held: quantise, back, and once more gives the same (the largest value of a block is 4 or 6 steps)."""
    x = torch.randn(77, 640, generator=gen(3), device="cuda")
    q, s = run_quantize(lib, x, fmt)
    y = torch.empty_like(x)
    lib.fp4_dequantize(q, s, y)
    v = ref.values(q, s, fmt, 640)
    assert bool((y.double() == v).all())
    # half a step of the values next to it: 1 of 6 steps between 4 and 6, rounded scales (NV) 1/16 more
    amax = ref.spread(ref.block_amax(x, fmt), 640, fmt)
    assert bool(((y.double() - x.double()).abs() <= (1 / 3 if fmt == MX else 1 / 6 + 1 / 16) * amax).all())


# ---- products --------------------------------------------------------------------------------------------------------------------

def operands(lib, rows, K, fmt, seed, lead=()):
    """Random codes and scales of a realistic spread, laid out for a product."""
    g = gen(seed)
    shape = (*lead, rows) if lead else rows
    q, s = lib.fp4_empty(shape, K, fmt)
    q.copy_(torch.randint(0, 256, q.shape, generator=g, device="cuda", dtype=torch.uint8))
    lo, hi = (120, 132) if fmt == MX else (40, 90)
    s.view(torch.uint8).copy_(torch.randint(lo, hi, s.shape, generator=g, device="cuda", dtype=torch.uint8))
    return q, s


def check_matmul(y, qa, sa, qb, sb, fmt, alpha=None):
    a, b = ref.values(qa, sa, fmt), ref.values(qb, sb, fmt)
    f = 1.0 if alpha is None else float(alpha)
    want, size = f * (a @ b.t()), abs(f) * (a.abs() @ b.abs().t())
    K = a.shape[1]
    half = torch.finfo(y.dtype).eps / 2
    err = ref.sum_error(K) * size
    bound = err + half * (want.abs() + err) + torch.finfo(y.dtype).smallest_normal * 2.0 ** -10
    off = (y.double() - want).abs()
    # from half a step beyond the largest number on (65504 + 16 in fp16) a result rounds to infinity
    most = torch.finfo(y.dtype).max
    top = most + 2.0 ** math.floor(math.log2(most)) * half
    off[y.isinf() & (want.abs() + err >= top) & (y.sign() == want.sign())] = 0.0
    assert bool((off <= bound).all()), (float((off / bound).max()), float(off.max()), float(want.abs().max()))


@FMT
@pytest.mark.parametrize("yt", WIDE, ids=str)
@pytest.mark.parametrize("rows,N,K", [(1, 128, 256), (1, 1, 32), (1, 300, 4096), (3, 130, 96), (16, 128, 288), (17, 257, 512), (33, 100, 1056), (64, 384, 2048),
                                      (65, 128, 64), (100, 200, 800), (129, 256, 256), (300, 515, 1120), (513, 1000, 320), (256, 256, 8192)])
def test_matmul(lib, rows, N, K, yt, fmt):
    qa, sa = operands(lib, rows, K, fmt, rows + K)
    qb, sb = operands(lib, N, K, fmt, N + K)
    alpha = factor(0.37 * 2.0 ** -8)
    y = torch.full((rows, N), 5.0, device="cuda", dtype=yt)
    lib.fp4_matmul(qa, sa, qb, sb, y, alpha=alpha)
    assert lib.fp4_status() == lib.OK
    check_matmul(y, qa, sa, qb, sb, fmt, alpha)


@FMT
@pytest.mark.parametrize("rows", [1, 5, 40, 140, 600])
def test_matmul_exact(lib, rows, fmt):
    """Whole numbers, scales of one and two: every sum is exact, so results are equal; each block of the reduction and row has values of its own."""
    N, K = 272, 736
    g = gen(rows)
    codes = [torch.randint(0, 16, (n, K), generator=g, device="cuda") for n in (rows, N)]
    (qa, sa), (qb, sb) = lib.fp4_empty(rows, K, fmt), lib.fp4_empty(N, K, fmt)
    one = 127 if fmt == MX else 56
    for c, q, s in ((codes[0], qa, sa), (codes[1], qb, sb)):
        q.copy_(ref.pack(c))
        s.view(torch.uint8).copy_(one + torch.randint(0, 2, s.shape, generator=g, device="cuda", dtype=torch.uint8) * (1 if fmt == MX else 8))
    y = torch.zeros(rows, N, device="cuda")
    lib.fp4_matmul(qa, sa, qb, sb, y)
    assert lib.fp4_status() == lib.OK
    assert torch.equal(y.double(), ref.values(qa, sa, fmt) @ ref.values(qb, sb, fmt).t())


@FMT
@pytest.mark.parametrize("mean", [1, 12, 90, 300, 800], ids=lambda m: "mean%d" % m)
def test_matmul_groups(lib, mean, fmt):
    """Ragged groups, empty ones at both ends and between, rows before the first and behind the last, offsets that fall or lie outside."""
    G, N, K = 9, 200, 352
    g = gen(mean)
    count = torch.randint(0, 2 * mean + 1, (G,), generator=g, device="cuda")
    count[0] = count[4] = count[8] = 0
    first = 3
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).int() + first
    rows = int(offsets[-1]) + 5
    qa, sa = operands(lib, rows, K, fmt, mean)
    qb, sb = operands(lib, N, K, fmt, mean + 1, (G,))
    alpha = torch.rand(G, generator=g, device="cuda") + 0.5
    for yt in (torch.bfloat16, torch.float32):
        y = torch.full((rows, N), 5.0, device="cuda", dtype=yt)
        lib.fp4_matmul(qa, sa, qb, sb, y, alpha=alpha, offsets=offsets)
        assert lib.fp4_status() == lib.OK
        at = offsets.tolist()
        assert bool((y[:first] == 5.0).all()) and bool((y[at[-1]:] == 5.0).all())
        for e in range(G):
            if at[e + 1] > at[e]:
                check_matmul(y[at[e]:at[e + 1]], qa[at[e]:at[e + 1]], sa[at[e]:at[e + 1]], qb[e], sb[e], fmt, alpha[e])
    if mean > 1:
        bad = offsets.clone()
        bad[3] = -7  # falls: as the largest before it
        bad[-1] = rows + 100
        y = torch.full((rows, N), 5.0, device="cuda")
        lib.fp4_matmul(qa, sa, qb, sb, y, offsets=bad)
        at = [max(0, min(v, rows)) for v in bad.tolist()]
        for i in range(1, G + 1):
            at[i] = max(at[i], at[i - 1])
        for e in range(G):
            if at[e + 1] > at[e]:
                check_matmul(y[at[e]:at[e + 1]], qa[at[e]:at[e + 1]], sa[at[e]:at[e + 1]], qb[e], sb[e], fmt)


@FMT
@pytest.mark.parametrize("yt,N,first,ld", [(torch.bfloat16, 1504, 0, 1504), (torch.float16, 1501, 3, 1511), (torch.bfloat16, 1530, 8, 1552), (torch.float32, 1476, 4, 1488),
                                           (torch.float32, 1501, 1, 1505)], ids=str)
def test_matmul_many_long_groups(lib, yt, N, first, ld, fmt):
    """Many groups and a long reduction: the weights take the accumulator's rows, a group's last tile has as many columns as there are rows left."""
    K, count = 4128, [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 159, 160, 161, 192, 224, 225, 0, 255, 256, 257, 288, 400, 513, 300, 100, 7, 140, 260, 90, 350, 16, 48,
                      200, 330, 30, 170, 0]
    G, g, before = len(count), gen(N), 5
    offsets = torch.tensor([0] + count, device="cuda").cumsum(0).int() + before
    rows = int(offsets[-1]) + 6
    qa, sa = operands(lib, rows, K, fmt, N)
    qb, sb = operands(lib, N, K, fmt, N + 1, (G,))
    alpha = torch.rand(G, generator=g, device="cuda") + 0.5
    whole = torch.full((rows, ld + 16), 5.0, device="cuda", dtype=yt)
    y = whole[:, first:first + N]
    lib.fp4_matmul(qa, sa, qb, sb, y, alpha=alpha, offsets=offsets)
    assert lib.fp4_status() == lib.OK
    at = offsets.tolist()
    for e in range(G):
        if count[e]:
            check_matmul(y[at[e]:at[e + 1]], qa[at[e]:at[e + 1]], sa[at[e]:at[e + 1]], qb[e], sb[e], fmt, alpha[e])
    assert bool((whole[:before] == 5.0).all()) and bool((whole[at[-1]:] == 5.0).all())
    assert bool((whole[:, :first] == 5.0).all()) and bool((whole[:, first + N:] == 5.0).all())
    bad = at[20] + 100  # a row with a NaN is NaN, and no other, also where its neighbours are another group's
    sa.view(torch.uint8)[bad, 3] = 255 if fmt == MX else 127
    again = whole.clone()
    lib.fp4_matmul(qa, sa, qb, sb, again[:, first:first + N], alpha=alpha, offsets=offsets)
    assert bool(again[bad, first:first + N].isnan().all())
    again[bad] = whole[bad]
    assert torch.equal(again, whole)


@FMT
@pytest.mark.parametrize("rows", [1, 30, 260])
def test_matmul_strides(lib, rows, fmt):
    """Rows of a and of its scales further apart, columns of y a part of a wider matrix, at places off the 16-byte grid."""
    N, K = 145, 160
    wide_q, wide_s = operands(lib, rows, K + 96, fmt, 5)
    qa, sa = wide_q[:, :K // 2], wide_s[:, :ref.nb(K, fmt)]
    qb, sb = operands(lib, N, K, fmt, 6)
    for yt in WIDE:
        for first, ld in ((0, 160), (1, 147), (3, 150), (8, 160)):
            whole = torch.full((rows, ld + 16), 5.0, device="cuda", dtype=yt)
            y = whole[:, first:first + N]
            lib.fp4_matmul(qa, sa, qb, sb, y)
            assert lib.fp4_status() == lib.OK
            check_matmul(y, qa, sa, qb, sb, fmt)
            assert bool((whole[:, :first] == 5.0).all()) and bool((whole[:, first + N:] == 5.0).all())


@FMT
@pytest.mark.parametrize("rows", [4, 200])
def test_matmul_nan_scales(lib, rows, fmt):
    """A block without a number makes its row (of a) or column (of b) NaN, and nothing else."""
    N, K = 150, 320
    qa, sa = operands(lib, rows, K, fmt, 7)
    qb, sb = operands(lib, N, K, fmt, 8)
    nan = 255 if fmt == MX else 127
    sa.view(torch.uint8)[rows - 1, 2], sb.view(torch.uint8)[77, 0] = nan, nan
    y = torch.zeros(rows, N, device="cuda")
    lib.fp4_matmul(qa, sa, qb, sb, y)
    want = torch.zeros(rows, N, dtype=torch.bool, device="cuda")
    want[rows - 1], want[:, 77] = True, True
    assert bool((y.isnan() == want).all())


@FMT
@pytest.mark.parametrize("rows", [2, 150])
def test_matmul_extreme_scales(lib, rows, fmt):
    """The smallest and the largest scales."""
    N, K = 70, 256
    qa, sa = operands(lib, rows, K, fmt, 9)
    qb, sb = operands(lib, N, K, fmt, 10)
    for ca, cb in ((0, 254), (254, 0), (100, 100), (160, 150)) if fmt == MX else ((1, 126), (126, 126), (1, 1), (0, 56), (7, 9)):
        sa.view(torch.uint8).fill_(ca)
        sb.view(torch.uint8).fill_(cb)
        y = torch.zeros(rows, N, device="cuda")
        lib.fp4_matmul(qa, sa, qb, sb, y)
        check_matmul(y, qa, sa, qb, sb, fmt)


def test_matmul_same_bits_twice(lib):
    """Cut reductions meet in a fixed order."""
    for rows in (1, 40, 300):
        qa, sa = operands(lib, rows, 4096, NV, 11)
        qb, sb = operands(lib, 384, 4096, NV, 12)
        ys = [torch.zeros(rows, 384, device="cuda") for _ in range(3)]
        for y in ys:
            lib.fp4_matmul(qa, sa, qb, sb, y)
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


# ---- expert layer ----------------------------------------------------------------------------------------------------------------

def layer(lib, hidden, inter, experts, fmt, seed):
    """Quantised weights of a layer with random ones of the usual size: (w1, its scales, w2, its scales, factors)."""
    g = gen(seed)
    out = []
    for shape, cols in (((experts, 2, inter), hidden), ((experts, hidden), inter)):
        w = torch.randn(*shape, cols, generator=g, device="cuda") / math.sqrt(cols)
        q, s = lib.fp4_empty(shape, cols, fmt)
        f = None
        if fmt == NV:
            f = w.abs().amax(tuple(range(1, w.dim()))) / 2688
        for e in range(experts):
            q1, s1 = lib.fp4_empty(math.prod(shape[1:]), cols, fmt)
            lib.fp4_quantize(w[e].reshape(-1, cols), q1, s1, global_scale=f[e:e + 1] if fmt == NV else None)
            q[e] = q1.view(*shape[1:], -1)
            s[e].view(torch.uint8).copy_(s1.view(torch.uint8).reshape(*shape[1:], -1))
        out += [q, s, f]
    return out


def run_experts(lib, x, ids, weights, w, fmt, gx=None, gh=None, extra=0):
    w1, s1, f1, w2, s2, f2 = w
    T, H = x.shape
    kind = {torch.float32: lib.F32, torch.float16: lib.F16, torch.bfloat16: lib.BF16}[x.dtype]
    n = lib.fp4_experts_workspace_bytes(H, w1.shape[2], w1.shape[0], ids.shape[1], T, fmt, kind)
    ws = torch.full((n + extra,), 0xFF, dtype=torch.uint8, device="cuda")
    y = torch.full_like(x, 9.0)
    lib.fp4_experts(x, ids, weights, w1, s1, w2, s2, y, ws, x_global=gx, w1_global=f1, h_global=gh, w2_global=f2)
    assert lib.fp4_status() == lib.OK
    assert bool((ws[n:] == 0xFF).all())
    return y


def check_experts(y, x, ids, weights, w, fmt, gx=None, gh=None):
    w1, s1, f1, w2, s2, f2 = w
    want, err = ref.experts(x, ids, weights, w1, s1, w2, s2, fmt, x.dtype, 1.0 if gx is None else float(gx), f1, 1.0 if gh is None else float(gh), f2)
    off = (y.double() - want).abs()
    assert bool((off <= err).all()), (float((off / err).max()), float(off.max()))
    # the bound allows for moved values anywhere; few move, so the whole is much nearer: within the rounding of y and a hundredth
    assert float(off.norm()) <= (torch.finfo(x.dtype).eps / 2 + 0.01) * float(want.norm())


def routes(T, experts, topk, seed):
    g = gen(seed)
    score = torch.rand(T, experts, generator=g, device="cuda")
    top = score.topk(topk, -1)
    return top.indices.int(), top.values / top.values.sum(-1, keepdim=True)


@FMT
@pytest.mark.parametrize("T,experts,topk,hidden,inter", [(1, 8, 2, 256, 128), (1, 4, 4, 32, 32), (2, 16, 1, 480, 96), (5, 8, 4, 544, 224), (16, 64, 4, 256, 160), (33, 8, 2, 384, 320),
                                                         (100, 6, 3, 288, 352), (300, 4, 2, 256, 256), (1000, 8, 2, 320, 96), (2000, 3, 2, 256, 128)])
@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float32], ids=str)
def test_experts(lib, T, experts, topk, hidden, inter, xt, fmt):
    w = layer(lib, hidden, inter, experts, fmt, T)
    x = torch.randn(T, hidden, generator=gen(T + 1), device="cuda").to(xt)
    ids, weights = routes(T, experts, topk, T + 2)
    gx, gh = (factor(6 / 2688), factor(9 / 2688)) if fmt == NV else (None, None)
    y = run_experts(lib, x, ids, weights, w, fmt, gx, gh, extra=64)
    check_experts(y, x, ids, weights, w, fmt, gx, gh)


@FMT
@pytest.mark.parametrize("T", [1, 6, 40, 700])
def test_experts_padded_batch(lib, T, fmt):
    """Ids that are no expert, tokens without any, an expert twice in a token, all tokens at one expert."""
    w = layer(lib, 256, 128, 5, fmt, T)
    x = torch.randn(T, 256, generator=gen(T), device="cuda").half()
    ids, weights = routes(T, 5, 3, T)
    ids[::3, 1] = -1
    ids[::4, 0] = 5
    ids[::5] = 1 << 30
    ids[1::5] = 2
    y = run_experts(lib, x, ids, weights, w, fmt)
    check_experts(y, x, ids, weights, w, fmt)
    assert bool((y[::5] == 0).all())


def test_experts_no_tokens(lib):
    w = layer(lib, 64, 32, 2, MX, 1)
    x = torch.zeros(0, 64, device="cuda")
    run_experts(lib, x, torch.zeros(0, 1, dtype=torch.int32, device="cuda"), torch.zeros(0, 1, device="cuda"), w, MX)


def test_layer_from_route_and_its_parts(lib):
    """Router, sort, quantisation, products of groups and weighted sum in a row, and the expert layer on the same route."""
    T, E, K, H, I, fmt = 90, 16, 4, 256, 256, NV
    w = layer(lib, H, I, E, fmt, 21)
    w1, s1, f1, w2, s2, f2 = w
    g = gen(22)
    logits = torch.randn(T, E, generator=g, device="cuda")
    weights, ids = torch.empty(T, K, device="cuda"), torch.empty(T, K, dtype=torch.int32, device="cuda")
    lib.route(lib.make_route_desc(E, K, score=lib.SCORE_SIGMOID), logits, weights, ids)
    x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    gx, gh = factor(6 / 2688), factor(9 / 2688)
    y = run_experts(lib, x, ids, weights, w, fmt, gx, gh)
    check_experts(y, x, ids, weights, w, fmt, gx, gh)

    offsets = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    rows, order = (torch.empty(T * K, dtype=torch.int32, device="cuda") for _ in range(2))
    lib.route_sort(ids, E, offsets, rows, order, torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))
    xq, xs = lib.fp4_empty(T * K, H, fmt)
    lib.fp4_quantize(x[order.long() // K], xq, xs, global_scale=gx)
    gate_up = torch.empty(T * K, 2 * I, device="cuda")
    both = s1.view(torch.uint8).reshape(E, 2 * I, -1)  # (a copy without gaps: rows of 16 scales)
    lib.fp4_matmul(xq, xs, w1.reshape(E, 2 * I, -1), both.view(s1.dtype), gate_up, alpha=f1 * gx, offsets=offsets)
    h = torch.nn.functional.silu(gate_up[:, :I]) * gate_up[:, I:]
    hq, hs = lib.fp4_empty(T * K, I, fmt)
    lib.fp4_quantize(h, hq, hs, global_scale=gh)
    parts = torch.empty(T * K, H, device="cuda")
    lib.fp4_matmul(hq, hs, w2, s2, parts, alpha=f2 * gh, offsets=offsets)
    out = torch.empty_like(x)
    lib.route_combine(parts, rows.reshape(T, K), weights, out)
    check_experts(out, x, ids, weights, w, fmt, gx, gh)


@FMT
def test_linear_layer(lib, fmt):
    """Weights and activations quantised and multiplied: as near to the product in 16 bits as 4 bits are."""
    g = gen(23)
    x, w = torch.randn(50, 1024, generator=g, device="cuda").bfloat16(), (torch.randn(300, 1024, generator=g, device="cuda") / 32).bfloat16()
    fx, fw = (None, None) if fmt == MX else ((v.abs().amax().float() / 2688).reshape(1) for v in (x, w))
    (xq, xs), (wq, ws) = lib.fp4_empty(50, 1024, fmt), lib.fp4_empty(300, 1024, fmt)
    lib.fp4_quantize(x, xq, xs, global_scale=fx)
    lib.fp4_quantize(w, wq, ws, global_scale=fw)
    y = torch.empty(50, 300, device="cuda", dtype=torch.bfloat16)
    lib.fp4_matmul(xq, xs, wq, ws, y, alpha=None if fmt == MX else fx * fw)
    want = x.double() @ w.double().t()
    # a value is off by a sixth of its block's largest at most (steps of a third of that, where nothing is beyond 6), NV by a sixteenth more
    # (its scale's rounding); normal values have their block's largest at 2 to 3 standard deviations, most steps are smaller, and errors of different
    # signs add up as the products do: a quarter of the size of the result covers two such operands
    assert float((y.double() - want).norm() / want.norm()) < 0.25


# ---- streams, graphs, sizes ------------------------------------------------------------------------------------------------------

@FMT
@pytest.mark.parametrize("rows", [3, 100, 400])
def test_matmul_streams_and_graph(lib, rows, fmt):
    """Two calls at once on two streams; a captured call replayed on new inputs."""
    K, N = 1024, 500
    sets = [(*operands(lib, rows, K, fmt, 30 + i), *operands(lib, N, K, fmt, 40 + i), torch.zeros(rows, N, device="cuda")) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, (qa, sa, qb, sb, y) in zip(streams, sets):
            lib.fp4_matmul(qa, sa, qb, sb, y, stream=st)
    torch.cuda.synchronize()
    for qa, sa, qb, sb, y in sets:
        check_matmul(y, qa, sa, qb, sb, fmt)
    qa, sa, qb, sb, y = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.fp4_matmul(qa, sa, qb, sb, y)
        lib.fp4_matmul(qa, sa, qb, sb, y)
    qa.copy_(sets[1][0])
    sa.view(torch.uint8).copy_(sets[1][1].view(torch.uint8))
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    check_matmul(y, qa, sa, qb, sb, fmt)
    assert lib.fp4_status() == lib.OK


@FMT
def test_quantize_stream_and_graph(lib, fmt):
    x = torch.randn(33, 512, generator=gen(31), device="cuda").bfloat16()
    q, s = lib.fp4_empty(33, 512, fmt)
    y = torch.empty_like(x)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    lib.fp4_quantize(x, q, s, stream=st)
    lib.fp4_dequantize(q, s, y, stream=st)
    torch.cuda.synchronize()
    check_quantize(x, fmt, q, s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.fp4_quantize(x, q, s)
        lib.fp4_dequantize(q, s, y)
    x.copy_(torch.randn(33, 512, generator=gen(32), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    check_quantize(x, fmt, q, s)
    assert bool((y.double() == ref.values(q, s, fmt, 512).to(y.dtype).double()).all())


@FMT
@pytest.mark.parametrize("tokens", [3, 60, 600])
def test_experts_graph(lib, tokens, fmt):
    """Two captured layers that share a workspace, replayed with other routes."""
    E, K, H, I = 16, 2, 256, 128
    x = torch.randn(tokens, H, generator=gen(33), device="cuda").bfloat16()
    ws = torch.empty(lib.fp4_experts_workspace_bytes(H, I, E, K, tokens, fmt), dtype=torch.uint8, device="cuda")
    ids, weights = routes(tokens, E, K, 34)
    nets = [(layer(lib, H, I, E, fmt, 35 + i), torch.empty_like(x)) for i in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for (w1, s1, f1, w2, s2, f2), y in nets:
            lib.fp4_experts(x, ids, weights, w1, s1, w2, s2, y, ws, w1_global=f1, w2_global=f2)
    for seed in (1, 2):
        i2, w2_ = routes(tokens, E, K, seed)
        ids.copy_(i2)
        weights.copy_(w2_)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        for w, y in nets:
            check_experts(y, x, ids, weights, w, fmt)
    assert lib.fp4_status() == lib.OK


@pytest.mark.parametrize("tokens", [2, 40])
def test_experts_two_streams(lib, tokens):
    """Two layers at once, each with a workspace of its own, and a large product on a third stream."""
    E, K, H, I, fmt = 16, 4, 512, 256, MX
    nets = []
    for i in range(2):
        x = torch.randn(tokens, H, generator=gen(50 + i), device="cuda").bfloat16()
        ws = torch.empty(lib.fp4_experts_workspace_bytes(H, I, E, K, tokens, fmt), dtype=torch.uint8, device="cuda")
        nets.append((x, *routes(tokens, E, K, 52 + i), layer(lib, H, I, E, fmt, 54 + i), torch.empty_like(x), ws, torch.cuda.Stream()))
    qa, sa = operands(lib, 2000, 2048, NV, 56)
    qb, sb = operands(lib, 2000, 2048, NV, 57)
    big, third = torch.empty(2000, 2000, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        lib.fp4_matmul(qa, sa, qb, sb, big, stream=third)
        for x, ids, weights, (w1, s1, f1, w2, s2, f2), y, ws, st in nets:
            lib.fp4_experts(x, ids, weights, w1, s1, w2, s2, y, ws, stream=st)
    torch.cuda.synchronize()
    for x, ids, weights, w, y, ws, st in nets:
        check_experts(y, x, ids, weights, w, fmt)
    check_matmul(big, qa, sa, qb, sb, NV)
    assert lib.fp4_status() == lib.OK


@FMT
@pytest.mark.parametrize("T,experts,topk", [(64, 64, 4), (65, 64, 4), (128, 64, 4), (129, 64, 4), (32, 8, 1), (33, 8, 1), (16, 1024, 32), (512, 1024, 1), (171, 700, 3)])
def test_experts_at_the_border_of_few(lib, T, experts, topk, fmt):
    """As many pairs as the two kernels for few tokens take, and one token more; very many experts."""
    w = layer(lib, 64, 32, experts, fmt, T)
    x = torch.randn(T, 64, generator=gen(T), device="cuda").half()
    ids, weights = routes(T, experts, topk, T)
    y = run_experts(lib, x, ids, weights, w, fmt, extra=256)
    check_experts(y, x, ids, weights, w, fmt)


def test_experts_strides(lib):
    """Rows of x and y further apart and off the 16-byte grid; every other token of a larger batch."""
    w = layer(lib, 160, 96, 6, NV, 60)
    w1, s1, f1, w2, s2, f2 = w
    for T in (3, 90):
        base = torch.randn(2 * T, 167, generator=gen(61), device="cuda").bfloat16()
        x = base[::2, 3:163]
        ids, weights = routes(T, 6, 2, 62)
        whole = torch.full((T, 171), 9.0, device="cuda", dtype=torch.bfloat16)
        y = whole[:, 5:165]
        ws = torch.empty(lib.fp4_experts_workspace_bytes(160, 96, 6, 2, T, NV), dtype=torch.uint8, device="cuda")
        lib.fp4_experts(x, ids, weights, w1, s1, w2, s2, y, ws, w1_global=f1, w2_global=f2)
        check_experts(y, x, ids, weights, w, NV)
        assert bool((whole[:, :5] == 9.0).all()) and bool((whole[:, 165:] == 9.0).all())


@pytest.mark.parametrize("T", [2, 200])
def test_experts_nan(lib, T):
    """A token with a NaN has a NaN everywhere (its block's scale has none), the others do not; an infinity likewise."""
    w = layer(lib, 128, 64, 4, MX, 63)
    x = torch.randn(T, 128, generator=gen(64), device="cuda")
    x[T - 1, 5] = math.nan
    if T > 2:
        x[7, 100] = math.inf
    ids, weights = routes(T, 4, 2, 65)
    y = run_experts(lib, x, ids, weights, w, MX)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[T - 1] = True
    if T > 2:
        bad[7] = True
    assert bool((y.isnan().all(1) == bad).all()) and bool((y.isnan().any(1) == bad).all())


@FMT
def test_many_groups(lib, fmt):
    """1024 groups of which a few have a row or two."""
    G, N, K = 1024, 40, 96
    count = torch.zeros(G, dtype=torch.long)
    count[[0, 5, 511, 512, 1023]] = torch.tensor([1, 2, 1, 3, 2])
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).int().cuda()
    rows = int(count.sum())
    qa, sa = operands(lib, rows, K, fmt, 66)
    qb, sb = operands(lib, N, K, fmt, 67, (G,))
    y = torch.zeros(rows, N, device="cuda")
    lib.fp4_matmul(qa, sa, qb, sb, y, offsets=offsets)
    at = offsets.tolist()
    for e in (0, 5, 511, 512, 1023):
        check_matmul(y[at[e]:at[e + 1]], qa[at[e]:at[e + 1]], sa[at[e]:at[e + 1]], qb[e], sb[e], fmt)


@FMT
@pytest.mark.parametrize("rows", [1, 70, 260])
def test_long_reduction(lib, rows, fmt):
    qa, sa = operands(lib, rows, 40000, fmt, 68)
    qb, sb = operands(lib, 130, 40000, fmt, 69)
    y = torch.zeros(rows, 130, device="cuda")
    lib.fp4_matmul(qa, sa, qb, sb, y)
    check_matmul(y, qa, sa, qb, sb, fmt)


@FMT
@pytest.mark.parametrize("cols", [512, 333])
def test_offsets_past_32_bits(lib, cols, fmt):
    """Rows more than 2^31 elements and bytes apart."""
    far = (1 << 31) + 96
    x = torch.zeros(far + cols, dtype=torch.bfloat16, device="cuda").as_strided((2, cols), (far, 1))
    x.copy_(torch.randn(2, cols, generator=gen(70), device="cuda"))
    q = torch.zeros(far + cols, dtype=torch.uint8, device="cuda").as_strided((2, (cols + 1) // 2), (far, 1))
    s = torch.zeros(far + cols, dtype=torch.uint8, device="cuda").as_strided((2, ref.nb(cols, fmt)), (far, 1)).view(ref.SCALE[fmt])
    lib.fp4_quantize(x, q, s)
    check_quantize(x, fmt, q, s)
    y = torch.zeros(far + cols, dtype=torch.bfloat16, device="cuda").as_strided((2, cols), (far, 1))
    lib.fp4_dequantize(q, s, y)
    assert bool((y.double() == ref.values(q, s, fmt, cols).to(y.dtype).double()).all())
    if cols == 512:
        b, sb = operands(lib, 100, 512, fmt, 71)
        out = torch.zeros(far + cols, dtype=torch.bfloat16, device="cuda").as_strided((2, 100), (far, 1))
        lib.fp4_matmul(q, s, b, sb, out)
        check_matmul(out, q, s, b, sb, fmt)


def test_very_many_rows(lib):
    """Very many short rows of an odd width."""
    x = torch.randn(1 << 12, 33, generator=gen(72), device="cuda").bfloat16()
    rows = 1 << 20
    big = x.repeat(rows >> 12, 1)
    q, s = torch.zeros(rows, 17, dtype=torch.uint8, device="cuda"), torch.zeros(rows, 3, dtype=torch.uint8, device="cuda").view(ref.SCALE[NV])
    lib.fp4_quantize(big, q, s)
    check_quantize(x, NV, q[-(1 << 12):], s[-(1 << 12):])
    assert torch.equal(q[:1 << 12], q[-(1 << 12):]) and torch.equal(s.view(torch.uint8)[:1 << 12], s.view(torch.uint8)[-(1 << 12):])


@pytest.mark.parametrize("form", [0, 1, 2])
def test_bounded_wait(lib, form):
    """A wait that cannot end gives up and is reported once; the device goes on."""
    lib.selftest_fp4_wait(form)
    assert lib.fp4_status() == lib.E_TIMEOUT
    assert lib.fp4_status() == lib.OK
    x = torch.ones(1, 32, device="cuda")
    q, s = lib.fp4_empty(1, 32, lib.MXFP4)
    lib.fp4_quantize(x, q, s)
    check_quantize(x, MX, q, s)
