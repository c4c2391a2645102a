"""8-bit float operators on the device against their definitions in 64 bits (fp8_ref)."""
import math

import pytest
import torch

import fp8_ref as ref

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
WIDE = [torch.float32, torch.float16, torch.bfloat16]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def poison(rows, cols, dtype, ld=None, value=7.0):
    """A matrix filled with a value, a view into wider rows if `ld` is given."""
    whole = torch.full((rows, ld or cols), value, device="cuda").to(dtype)
    return whole, whole[:, :cols]


def same8(got, want):
    """8-bit results equal in value, NaN in the same places."""
    got = got.double()
    return bool((got.isnan() == want.isnan()).all()) and bool((torch.where(got.isnan(), 0.0, got) == torch.where(want.isnan(), 0.0, want)).all())


def run_quantize(lib, x, dtype, block, ldq=None, lds=None):
    rows, cols = x.shape
    wq, q = poison(rows, cols, dtype, ldq, 2.0)
    ws, s = poison(-(-rows // block), ref.nb(cols), torch.float32, lds, -3.0)
    lib.fp8_quantize(x, q, s, block_rows=block)
    torch.cuda.synchronize()
    assert bool((wq[:, cols:].float() == 2.0).all()) and bool((ws[:, ref.nb(cols):] == -3.0).all())
    return q, s


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [E4, E5], ids=["e4m3", "e5m2"])
@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 1), (3, 127), (5, 129), (64, 384), (130, 1000), (257, 128), (1, 8192)])
def test_quantize(lib, rows, cols, xt, dtype, block):
    # 16-bit numbers in every type: x * F / amax is then free of rounding up to the last step, so results are equal
    x = (torch.randn(rows, cols, generator=gen(rows + cols), device="cuda") * 3).bfloat16().to(xt)
    q, s = run_quantize(lib, x, dtype, block)
    want, scale = ref.quantize(x, dtype, block)
    assert same8(q, want)
    assert bool(((s.double() - scale).abs() <= 2.0 ** -24 * scale).all())


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_full_float(lib, block):
    """fp32 numbers of 24 bits: only values closer to a border than the two roundings before it may fall to its other side."""
    x = torch.randn(200, 777, generator=gen(1), device="cuda")
    q, s = run_quantize(lib, x, E4, block)
    want, _ = ref.quantize(x, E4, block)
    v = x.double() * 448 / ref.spread(ref.amax_of(x, block), 200, 777, block)
    low, high = ref.round8(v * (1 - 2.0 ** -23), E4), ref.round8(v * (1 + 2.0 ** -23), E4)
    assert bool(((q.double() == low) | (q.double() == high)).all())
    assert float((q.double() != want).double().mean()) < 1e-4


def test_quantize_ties(lib):
    """Half way between two values: to the even one, for every border of the type and both signs."""
    v = torch.arange(0, 256, dtype=torch.uint8).view(E4).double()
    v = v[v.isfinite() & (v >= 0)].sort().values
    mid = (v[:-1] + v[1:]) / 2
    x = torch.cat([mid, -mid, torch.tensor([448.0])]).float().cuda()
    x = torch.nn.functional.pad(x, (0, -x.numel() % 128)).reshape(-1, 128).clone()
    x[:, 127] = 448.0  # every block has the scale 1
    for f in (1.0, 2.0 ** -30, 1.5 * 2.0 ** 20, 2.0 ** 100):
        q, s = run_quantize(lib, x * f, E4, 1)
        want, _ = ref.quantize(x * f, E4, 1)
        assert same8(q, want)


@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_special_values(lib, block, xt):
    x = torch.randn(140, 520, generator=gen(3), device="cuda").to(xt)
    x[0] = 0.0
    x[1, 5] = math.nan
    x[2, 130] = math.inf
    x[3, 400] = -math.inf
    x[4] = 1e-38
    x[5] *= 1e37
    x[6] *= 2.0 ** -101
    x[7, :128] = math.nan
    x[8, 0], x[8, 1] = 3.3e38, -3.3e38
    q, s = run_quantize(lib, x, E4, block)
    want, scale = ref.quantize(x, E4, block)
    assert same8(q, want)
    finite = scale.isfinite()
    assert bool((s.isinf() == scale.isinf()).all())
    assert bool(((s.double() - scale).abs()[finite] <= 2.0 ** -24 * scale[finite]).all())


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("dtype", [E4, E5], ids=["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,cols,first", [(300, 777, 0), (300, 640, 3), (9000, 2000, 0)])
def test_quantize_special_values_among_others(lib, rows, cols, first, block, dtype, xt):
    """Rows off the 16-byte grid and very many blocks: NaN, infinities, zeros of both signs, the smallest and the largest values."""
    x = torch.randn(rows, first + cols, generator=gen(4), device="cuda").bfloat16().to(xt)[:, first:]
    tiny, large = torch.finfo(xt).tiny, torch.finfo(xt).max
    spots = torch.rand(rows, cols, generator=gen(5), device="cuda")
    x[1::128][spots[1::128] < 2e-3] = math.nan
    x[200::256][spots[200::256] < 2e-3] = math.inf
    x[201::256][spots[201::256] < 1e-3] = -math.inf
    x[130::512] = -0.0
    x[131::512] = tiny / 4
    x[132::512][spots[132::512] < 0.01] = -large
    q, s = run_quantize(lib, x, dtype, block)
    want, scale = ref.quantize(x, dtype, block)
    finite = scale.isfinite()
    assert bool((s.isinf() == scale.isinf()).all()) and bool((s.isnan() == scale.isnan()).all())
    assert bool(((s.double() - scale).abs()[finite] <= 2.0 ** -24 * scale[finite]).all())
    assert same8(q, want)


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_strides_and_alignment(lib, block):
    base = torch.randn(70, 1024, generator=gen(4), device="cuda").bfloat16()
    for x, ldq, lds in [(base[:, 3:500], 511, 9), (base[::2, 8:520], 528, None), (base[:, :512], 515, 4), (base[:1, 1:130], None, None)]:
        q, s = run_quantize(lib, x, E4, block, ldq, lds)
        assert same8(q, ref.quantize(x, E4, block)[0])


def test_quantize_no_rows(lib):
    lib.fp8_quantize(torch.zeros(0, 64, device="cuda"), torch.zeros(0, 64, device="cuda").to(E4), torch.zeros(0, 1, device="cuda"))


# ---- products --------------------------------------------------------------------------------------------------------------------


def whole_numbers(g, rows, K, dtype, block, groups=None):
    """Small whole numbers and scales that are powers of two: every partial sum fits fp32, so results are exact."""
    shape = (rows, K) if groups is None else (groups, rows, K)
    q = torch.randint(-3, 4, shape, generator=g, device="cuda").float().to(dtype)
    sshape = (-(-rows // block), ref.nb(K))
    s = 2.0 ** torch.randint(-2, 3, sshape if groups is None else (groups,) + sshape, generator=g, device="cuda").float()
    return q, s


SHAPES = [(1, 1, 16), (1, 8192, 128), (1, 300, 8192), (2, 128, 256), (7, 129, 144), (16, 64, 4096), (17, 257, 400), (33, 1000, 1040), (64, 128, 2048),
          (65, 640, 272), (100, 127, 128), (128, 512, 512), (129, 4096, 160), (200, 384, 1536), (255, 255, 2064), (256, 2048, 256), (300, 130, 640),
          (513, 777, 304), (1024, 1024, 1024), (1500, 264, 128)]


@pytest.mark.parametrize("rows,N,K", SHAPES)
def test_matmul_exact(lib, rows, N, K):
    g = gen(rows * 7 + N + K)
    a, sa = whole_numbers(g, rows, K, E4, 1)
    b, sb = whole_numbers(g, N, K, E4, 128)
    _, y = poison(rows, N, torch.float32)
    lib.fp8_matmul(a, sa, b, sb, y)
    torch.cuda.synchronize()
    assert lib.fp8_status() == lib.OK
    assert torch.equal(y.double(), ref.matmul(a, sa, b, sb))


@pytest.mark.parametrize("yt", WIDE, ids=str)
@pytest.mark.parametrize("at,bt", [(E4, E4), (E5, E4), (E4, E5), (E5, E5)], ids=["e4e4", "e5e4", "e4e5", "e5e5"])
@pytest.mark.parametrize("rows,N,K", [(1, 1024, 2048), (5, 333, 208), (48, 520, 4112), (150, 1030, 528), (700, 650, 2000)])
def test_matmul_types(lib, rows, N, K, at, bt, yt):
    g = gen(rows)
    a, sa = ref.quantize(torch.randn(rows, K, generator=g, device="cuda"), at)
    b, sb = ref.quantize(torch.randn(N, K, generator=g, device="cuda"), bt, 128)
    a, sa, b, sb = a.to(at), sa.float(), b.to(bt), sb.float()
    _, y = poison(rows, N, yt)
    lib.fp8_matmul(a, sa, b, sb, y)
    want = ref.matmul(a, sa, b, sb)
    off = (y.double() - want).abs()
    sums = ref.sum_error(K) * ref.size_of_sums(a, sa, b, sb)
    half = torch.finfo(yt).eps / 2
    assert bool((off <= sums + half * (want.abs() + sums)).all())
    # and on the whole far nearer than the worst case: rounding errors of a sum grow with its square root
    assert float(off.norm() / want.norm()) < half + 2.0 ** -23 * math.sqrt(K)
    assert lib.fp8_status() == lib.OK


@pytest.mark.parametrize("yt", WIDE, ids=str)
@pytest.mark.parametrize("rows,N,K", [(3, 200, 256), (40, 129, 128), (300, 520, 384), (700, 300, 128)])
def test_matmul_strides(lib, rows, N, K, yt):
    g = gen(rows)
    a, sa = whole_numbers(g, rows, K + 64, E4, 1)
    b, sb = whole_numbers(g, N, K, E4, 128)
    a, sa = a[:, 16:16 + K], sa[:, :ref.nb(K)]
    for ldy in (N, N + 3, N + 24):
        whole, y = poison(rows, N, yt, ldy)
        lib.fp8_matmul(a, sa, b, sb, y)
        assert torch.equal(y.double(), ref.matmul(a, sa, b, sb).to(yt).double())
        assert bool((whole[:, N:].float() == 7.0).all())
    for n in (N - 1, N - 2, N - 93, N - 101):  # rows on the 16-byte grid that end off it
        whole, _ = poison(rows, N // 8 * 8 + 16, yt)
        lib.fp8_matmul(a, sa, b[:n], sb[:ref.nb(n)], whole[:, :n])
        assert torch.equal(whole[:, :n].double(), ref.matmul(a, sa, b[:n], sb[:ref.nb(n)]).to(yt).double())
        assert bool((whole[:, n:].float() == 7.0).all())
    for first in (1, 4, 7):  # results that start off the 16-byte grid
        whole, _ = poison(rows, N + 8, yt)
        lib.fp8_matmul(a, sa, b, sb, whole[:, first:first + N])
        assert torch.equal(whole[:, first:first + N].double(), ref.matmul(a, sa, b, sb).to(yt).double())
        assert bool((whole[:, :first].float() == 7.0).all()) and bool((whole[:, first + N:].float() == 7.0).all())


def group_sizes(kind, groups, rows, g):
    if kind == "even":
        n = torch.full((groups,), rows // groups)
    elif kind == "one":
        n = torch.zeros(groups, dtype=torch.long)
        n[groups // 2] = rows
    elif kind == "single rows":
        n = torch.ones(groups, dtype=torch.long) if groups <= rows else (torch.arange(groups) % 2 == 0).long()
    elif kind == "none":
        n = torch.zeros(groups, dtype=torch.long)
    else:
        n = torch.randint(0, 2 * rows // groups + 1, (groups,), generator=torch.Generator().manual_seed(groups))
        n[groups // 3] = 0
        while int(n.sum()) > rows:
            n = n * 3 // 4
    return torch.nn.functional.pad(n.cumsum(0), (1, 0)).int().cuda()


@pytest.mark.parametrize("kind", ["even", "one", "single rows", "none", "ragged"])
@pytest.mark.parametrize("groups,rows,N,K", [(2, 10, 64, 128), (8, 64, 300, 512), (33, 70, 128, 272), (5, 1300, 384, 256), (64, 4000, 200, 128), (1000, 1500, 16, 32)])
def test_matmul_groups(lib, groups, rows, N, K, kind):
    g = gen(groups + rows)
    a, sa = whole_numbers(g, rows, K, E4, 1)
    b, sb = whole_numbers(g, N, K, E4, 128, groups)
    offsets = group_sizes(kind, groups, rows, g)
    _, y = poison(rows, N, torch.float32)
    lib.fp8_matmul(a, sa, b, sb, y, offsets=offsets)
    torch.cuda.synchronize()
    assert lib.fp8_status() == lib.OK
    at = offsets.tolist()
    want = torch.full((rows, N), 7.0, dtype=torch.float64, device="cuda")  # rows of no group stay
    for e in range(groups):
        if at[e + 1] > at[e]:
            want[at[e]:at[e + 1]] = ref.matmul(a[at[e]:at[e + 1]], sa[at[e]:at[e + 1]], b[e], sb[e])
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("rows", [9, 700])
def test_matmul_offsets_outside(lib, rows):
    """Offsets below zero or past the rows are taken as the nearest valid ones, a falling one as the largest before it."""
    g = gen(5)
    a, sa = whole_numbers(g, rows, 128, E4, 1)
    b, sb = whole_numbers(g, 96, 128, E4, 128, 4)
    _, y = poison(rows, 96, torch.float32)
    lib.fp8_matmul(a, sa, b, sb, y, offsets=torch.tensor([-5, 3, 2, 6, rows + 1000], dtype=torch.int32, device="cuda"))
    want = torch.full((rows, 96), 7.0, dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate([(0, 3), (3, 3), (3, 6), (6, rows)]):
        if hi > lo:
            want[lo:hi] = ref.matmul(a[lo:hi], sa[lo:hi], b[e], sb[e])
    assert torch.equal(y.double(), want)


def test_matmul_nan_rows_stay_apart(lib):
    """A NaN in one row, an infinite scale in another: the other rows are not touched by them."""
    g = gen(6)
    for rows in (20, 400):
        a, sa = whole_numbers(g, rows, 384, E4, 1)
        b, sb = whole_numbers(g, 200, 384, E4, 128)
        a.view(torch.uint8)[3, 100] = 0x7F
        sa[7, 1] = math.inf
        _, y = poison(rows, 200, torch.bfloat16)
        lib.fp8_matmul(a, sa, b, sb, y)
        keep = [i for i in range(rows) if i not in (3, 7)]
        assert torch.equal(y.double()[keep], ref.matmul(a[keep], sa[keep], b, sb).bfloat16().double())
        assert bool(y[3].isnan().all()) and not bool(y[7].isfinite().any())


@pytest.mark.parametrize("rows", [4, 600])
def test_matmul_streams_and_graph(lib, rows):
    """Two calls at once on two streams; a captured call replayed on new inputs."""
    g = gen(8)
    sets = []
    for _ in range(2):
        a, sa = whole_numbers(g, rows, 1024, E4, 1)
        b, sb = whole_numbers(g, 1000, 1024, E4, 128)
        sets.append((a, sa, b, sb, poison(rows, 1000, torch.float32)[1], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for a, sa, b, sb, y, st in sets:
            lib.fp8_matmul(a, sa, b, sb, y, stream=st)
    torch.cuda.synchronize()
    for a, sa, b, sb, y, _ in sets:
        assert torch.equal(y.double(), ref.matmul(a, sa, b, sb))
    a, sa, b, sb, y, st = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.fp8_matmul(a, sa, b, sb, y)
    a.copy_(sets[1][0])
    sa.copy_(sets[1][1])
    y.fill_(5.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.double(), ref.matmul(a, sa, b, sb))
    assert lib.fp8_status() == lib.OK


@pytest.mark.parametrize("rows", [63, 64, 65, 127, 129, 191, 193, 256, 257, 319, 384, 385, 512, 513, 769])
@pytest.mark.parametrize("N,K", [(128, 2048), (1000, 512), (4096, 128)])
def test_matmul_row_counts(lib, rows, N, K):
    """Row counts round which the kernel, its tile or the cut of the reduction change."""
    g = gen(rows)
    a, sa = whole_numbers(g, rows, K, E4, 1)
    b, sb = whole_numbers(g, N, K, E4, 128)
    _, y = poison(rows, N, torch.bfloat16)
    lib.fp8_matmul(a, sa, b, sb, y)
    assert torch.equal(y.double(), ref.matmul(a, sa, b, sb).bfloat16().double())
    assert lib.fp8_status() == lib.OK


def test_tensors_of_more_than_32_bits(lib):
    """Offsets past 2^31 elements: the last rows of a result, of an input and of their scales."""
    rows, N = 280000, 8192
    g = gen(10)
    a, sa = whole_numbers(g, rows, 128, E4, 1)
    b, sb = whole_numbers(g, N, 128, E4, 128)
    y = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda")
    lib.fp8_matmul(a, sa, b, sb, y)
    for lo in (0, 262100, rows - 300):
        want = ref.matmul(a[lo:lo + 300], sa[lo:lo + 300], b, sb).bfloat16()
        assert torch.equal(y[lo:lo + 300], want)
    q, s = torch.empty(rows, N, dtype=torch.uint8, device="cuda").view(E4), torch.empty(rows, N // 128, device="cuda")
    lib.fp8_quantize(y, q, s)
    for lo in (0, 262100, rows - 300):
        assert same8(q[lo:lo + 300], ref.quantize(y[lo:lo + 300], E4)[0])
    # 16 input rows far apart, few results
    wide = q.view(torch.uint8).view(-1)[: 16 * (1 << 27)].view(E4).view(16, 1 << 27)[:, :256]
    sw = torch.ones(16, 2, device="cuda")
    b2, s2 = whole_numbers(g, 100, 256, E4, 128)
    small = torch.empty(16, 100, device="cuda")
    lib.fp8_matmul(wide, sw, b2, s2, small)
    want = ref.matmul(wide, sw, b2, s2)
    bound = ref.sum_error(256) * ref.size_of_sums(wide, sw, b2, s2)
    assert bool(((small.double() - want).abs() <= bound + 2.0 ** -24 * want.abs()).all())
    assert lib.fp8_status() == lib.OK


def test_matmul_repeats_bit_for_bit(lib):
    g = gen(9)
    for rows, N, K in [(1, 2048, 8192), (48, 1030, 4112), (600, 700, 2048)]:
        a, sa = ref.quantize(torch.randn(rows, K, generator=g, device="cuda"), E4)
        b, sb = ref.quantize(torch.randn(N, K, generator=g, device="cuda"), E4, 128)
        a, sa, b, sb = a.to(E4), sa.float(), b.to(E4), sb.float()
        ys = [poison(rows, N, torch.float32)[1] for _ in range(4)]
        for y in ys:
            lib.fp8_matmul(a, sa, b, sb, y)
        assert all(torch.equal(y, ys[0]) for y in ys)


# ---- routing ---------------------------------------------------------------------------------------------------------------------


def run_route(lib, x, topk, kind="softmax", groups=1, topk_groups=1, group_score="max", renormalise=True, scale=1.0, bias=None):
    d = lib.make_route_desc(x.shape[1], topk, lib.SCORE_SOFTMAX if kind == "softmax" else lib.SCORE_SIGMOID, groups, topk_groups,
                            lib.GROUP_MAX if group_score == "max" else lib.GROUP_TOP2, renormalise, scale)
    w = torch.full((x.shape[0], topk), -1.0, device="cuda")
    ids = torch.full((x.shape[0], topk), -9, dtype=torch.int32, device="cuda")
    lib.route(d, x, w, ids, bias=bias)
    torch.cuda.synchronize()
    return w, ids


def check_route(lib, x, topk, **kw):
    w, ids = run_route(lib, x, topk, **kw)
    rw, rids = ref.route(x, topk, **kw)
    wrong = (ids.cpu() != rids).any(-1).nonzero().flatten().tolist()
    assert not wrong, (wrong, ids[wrong[0]], rids[wrong[0]])
    # a few roundings to 32 bits of exp, quotient, sum and product: eight units of rounding
    off = ~((w.cpu().double() - rw).abs() <= 8 * 2.0 ** -24 * rw.abs() + 1e-40)
    assert not bool(off.any()), (off.nonzero()[0], w.cpu()[off][0], rw[off][0])


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,topk,groups,topk_groups,group_score", [
    (1, 1, 1, 1, 1, "max"), (1, 64, 4, 1, 1, "max"), (5, 8, 8, 1, 1, "max"), (33, 60, 6, 1, 1, "max"), (7, 128, 8, 4, 2, "max"),
    (50, 256, 8, 8, 4, "top2"), (9, 512, 10, 8, 3, "top2"), (3, 1024, 32, 32, 5, "top2"), (4, 33, 5, 3, 2, "top2"), (6, 32, 3, 32, 4, "top2"),
    (11, 160, 8, 1, 1, "max"), (130, 96, 2, 8, 8, "max"), (5, 160, 6, 8, 3, "top2"), (4, 1018, 9, 2, 1, "top2"), (6, 1000, 5, 5, 3, "max"),
    (3, 200, 4, 25, 20, "top2")])
def test_route(lib, tokens, experts, topk, groups, topk_groups, group_score, kind, xt):
    g = gen(tokens + experts)
    x = (torch.randn(tokens, experts, generator=g, device="cuda") * 2).to(xt)
    bias = torch.randn(experts, generator=g, device="cuda") * 0.1
    for b in (None, bias):
        for renormalise, scale in ((True, 1.0), (False, 2.5)):
            check_route(lib, x, topk, kind=kind, groups=groups, topk_groups=topk_groups, group_score=group_score, renormalise=renormalise,
                        scale=scale, bias=b)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_route_special_rows(lib, kind, groups):
    """Rows that a mask empties, infinities, NaN, the type's lowest value, equal scores."""
    x = torch.randn(14, 64, generator=gen(12), device="cuda")
    x[0] = -math.inf
    x[1, 3:] = -math.inf
    x[2, 17] = math.nan
    x[3, 40] = math.inf
    x[4, 40], x[4, 9] = math.inf, math.inf
    x[5] = torch.finfo(torch.float32).min
    x[6] = 0.0
    x[7] = math.nan
    x[8, ::2] = x[8, 1::2]
    x[9] = 200.0 + torch.arange(64, device="cuda") % 3
    x[10] = -200.0 - torch.arange(64, device="cuda") % 3
    x[11, 5:] = torch.finfo(torch.float32).min
    x[12] = torch.round(x[12])
    bias = torch.zeros(64, device="cuda")
    bias[50] = -math.inf
    bias[20] = 0.25
    for b in (None, bias):
        check_route(lib, x, 6, kind=kind, groups=groups, topk_groups=min(groups, 2), bias=b)


@pytest.mark.parametrize("experts,groups", [(64, 1), (64, 4), (60, 3), (256, 8)])
def test_route_special_bias(lib, experts, groups):
    """Biases that take experts out, put them first or are NaN."""
    x = torch.randn(40, experts, generator=gen(15), device="cuda")
    bias = torch.randn(experts, generator=gen(16), device="cuda") * 0.1
    bias[::3] = -math.inf
    bias[1::5] = math.nan
    bias[2] = math.inf
    for kind in ("softmax", "sigmoid"):
        check_route(lib, x, 6, kind=kind, groups=groups, topk_groups=min(groups, 2), bias=bias)
    bias[:] = math.nan
    check_route(lib, x, 6, kind="sigmoid", groups=groups, topk_groups=min(groups, 2), bias=bias)


def test_route_near_scores_are_told_apart(lib):
    """Choices that differ by less than 32 bits can hold: the larger one is taken."""
    x = torch.zeros(64, 32, device="cuda")
    bias = torch.full((32,), 0.25, device="cuda")
    bias[31] = 0.25 + 2.0 ** -25  # s + bias = 0.75 + 2^-25 is 0.75 in 32 bits
    w, ids = run_route(lib, x, 2, kind="sigmoid", bias=bias)
    assert ids.tolist() == [[31, 0]] * 64
    y = torch.randn(200, 64, generator=gen(13), device="cuda") * 0.01
    near = y[:, :1] + torch.arange(64, device="cuda") * 2.0 ** -22  # neighbouring logits
    check_route(lib, near, 5, kind="sigmoid", bias=torch.full((64,), 0.5, device="cuda"))


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,topk,groups,topk_groups,group_score", [
    (400, 256, 8, 8, 4, "top2"), (401, 256, 15, 1, 1, "max"), (411, 33, 5, 1, 1, "max"), (397, 64, 6, 16, 5, "top2"), (501, 64, 3, 4, 2, "max"),
    (397, 240, 8, 5, 2, "top2"), (399, 96, 6, 4, 1, "max"), (300, 512, 16, 8, 4, "max")])
def test_route_ties_among_others(lib, tokens, experts, topk, groups, topk_groups, group_score, kind, xt):
    """Every third token has equal and nearly equal logits, so that neighbouring tokens need different looks."""
    g = gen(tokens + experts)
    x = torch.randn(tokens, experts, generator=g, device="cuda") * 2
    x[::3] = torch.round(x[::3]) + torch.arange(experts, device="cuda") % 4 * 2.0 ** -21
    x = x.to(xt)
    bias = torch.randn(experts, generator=g, device="cuda") * 0.1
    bias[::2] = 0.125
    for b in (None, bias):
        for renormalise, scale in ((True, 1.0), (False, 2.5)):
            check_route(lib, x, topk, kind=kind, groups=groups, topk_groups=topk_groups, group_score=group_score, renormalise=renormalise,
                        scale=scale, bias=b)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups", [(64, 1), (64, 4), (256, 8)])
def test_route_special_rows_among_others(lib, kind, experts, groups):
    """Emptied rows, infinities, NaN and ties beside ordinary tokens, and biases of the same kinds."""
    x = torch.randn(143, experts, generator=gen(17), device="cuda")
    x[0::14] = -math.inf
    x[1::14, 3:] = -math.inf
    x[2::14, 17] = math.nan
    x[4::14, 9::31] = math.inf
    x[5::14] = torch.finfo(torch.float32).min
    x[7::14] = 0.0
    x[8::14] = math.nan
    x[11::14] = -200.0 - torch.arange(experts, device="cuda") % 3
    bias = torch.randn(experts, generator=gen(18), device="cuda") * 0.1
    some = bias.clone()
    some[::3], some[1::5], some[2] = -math.inf, math.nan, math.inf
    for b in (None, bias, some):
        check_route(lib, x, 6, kind=kind, groups=groups, topk_groups=min(groups, 2), bias=b)


@pytest.mark.parametrize("experts", [885, 1024])
def test_route_weights_of_many_experts(lib, experts):
    """Sums over a whole row of like terms: their roundings stay few."""
    for seed in range(8):
        x = torch.rand(400, experts, generator=gen(40 + seed), device="cuda") * 0.5 ** seed
        check_route(lib, x, 5, kind="softmax", renormalise=False, scale=2.5)
        check_route(lib, x, 5, kind="softmax", renormalise=False, bias=x[0])


def test_route_equal_runs(lib):
    """Runs whose best logits are equal: the first ones are kept, in whatever place their best ones stand."""
    x = torch.zeros(40, 256, device="cuda")
    for g in range(8):
        x[torch.arange(40), 32 * g + (torch.arange(40, device="cuda") * (7 - g)) % 32] = 5.0
    for xt in WIDE:
        for kind in ("softmax", "sigmoid"):
            for score in ("max", "top2"):
                check_route(lib, x.to(xt), 4, kind=kind, groups=8, topk_groups=3, group_score=score)


def test_route_signed_zeros(lib):
    """-0 and +0 are equal."""
    x = torch.tensor([1.0, -1.0], device="cuda")[torch.randint(0, 2, (60, 96), generator=gen(21), device="cuda")] * 0.0
    x[::2, 70] = 1.0
    for xt in WIDE:
        for kind in ("softmax", "sigmoid"):
            check_route(lib, x.to(xt), 4, kind=kind)
            check_route(lib, x.to(xt), 4, kind=kind, groups=3, topk_groups=1)
            check_route(lib, x.to(xt), 4, kind=kind, bias=-x[0])


@pytest.mark.parametrize("experts,groups", [(64, 8), (64, 32), (60, 20), (60, 30), (256, 8), (256, 32), (96, 24)])
def test_route_runs_with_infinite_biases(lib, experts, groups):
    """Runs that a bias empties or puts first, in part and as a whole: sums of +inf and -inf are the lowest."""
    x = torch.randn(60, experts, generator=gen(22), device="cuda")
    size = experts // groups
    for seed in range(8):
        pick = torch.randint(0, 3, (experts,), generator=gen(30 + seed), device="cuda")
        bias = torch.tensor([0.125, math.inf, -math.inf], device="cuda")[pick]
        if seed % 2:
            bias[pick == 0] = math.nan
        if seed == 4:
            bias[::5] = torch.finfo(torch.float32).min
        for kind in ("softmax", "sigmoid"):
            check_route(lib, x, min(4, 3 * size), kind=kind, groups=groups, topk_groups=3, group_score="top2", bias=bias)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_weights_of_small_scores(lib, kind):
    """A bias or a run that takes experts whose scores 32 bits hardly hold or do not hold."""
    base = torch.tensor([50.0, -20.0, -88.0, -95.0, -100.0, -120.0, -600.0, -1500.0], device="cuda")
    x = torch.cat([base[:, None] + torch.randn(8, 32, generator=gen(19), device="cuda"), torch.randn(8, 32, generator=gen(20), device="cuda") * 40], 1)
    x[:, 40] = 60.0
    bias = torch.zeros(64, device="cuda")
    bias[:16] = 4.0
    for renormalise in (True, False):
        check_route(lib, x, 5, kind=kind, renormalise=renormalise, bias=bias)
        check_route(lib, x, 5, kind=kind, renormalise=renormalise, groups=2, topk_groups=1, bias=bias)


def test_route_strided_logits(lib):
    whole = torch.randn(20, 100, generator=gen(14), device="cuda")
    check_route(lib, whole[::2, 7:71], 4, kind="softmax")


@pytest.mark.parametrize("pairs,experts", [((1, 1), 1), ((1, 4), 64), ((37, 3), 7), ((256, 4), 64), ((300, 8), 256), ((5000, 2), 33), ((3000, 8), 1024),
                                           ((16384, 4), 9), ((70001, 1), 40), ((90000, 3), 130)])
def test_route_sort(lib, pairs, experts):
    g = gen(experts)
    ids = torch.randint(-2, experts + 2, pairs, generator=g, device="cuda").int()
    n = ids.numel()
    offsets = torch.full((experts + 1,), -9, dtype=torch.int32, device="cuda")
    rows = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    order = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, lib.route_sort_workspace_bytes(n, experts)), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        lib.route_sort(ids, experts, offsets, rows, order, ws)
    ro, rr, rorder = ref.sort(ids, experts)
    assert torch.equal(offsets.cpu(), ro) and torch.equal(rows.cpu(), rr)
    assert torch.equal(order.cpu()[:rorder.numel()], rorder) and bool((order[rorder.numel():] == -9).all())


@pytest.mark.parametrize("yt", WIDE, ids=str)
@pytest.mark.parametrize("ot", WIDE, ids=str)
@pytest.mark.parametrize("tokens,topk,cols", [(1, 1, 16), (5, 4, 1000), (40, 8, 2048), (3, 2, 7)])
def test_route_combine(lib, tokens, topk, cols, yt, ot):
    g = gen(cols)
    y = torch.randn(tokens * topk, cols + 8, generator=g, device="cuda").to(yt)[:, :cols]
    rows = torch.randperm(tokens * topk, generator=g, device="cuda").int().reshape(tokens, topk)
    rows[0, 0] = -1
    if tokens > 2:
        rows[2] = -1
        rows[1, 0] = 1 << 30  # no row of y
    w = torch.rand(tokens, topk, generator=g, device="cuda")
    whole, out = poison(tokens, cols, ot, cols + 5)
    lib.route_combine(y, rows, w, out)
    on = (rows >= 0) & (rows < tokens * topk)
    terms = torch.where(on, w, 0.0).double()[:, :, None] * y.double()[torch.where(on, rows, 0).long()]
    want, size = terms.sum(1), terms.abs().sum(1)
    half = torch.finfo(ot).eps / 2
    assert bool(((out.double() - want).abs() <= topk * 2.0 ** -24 * size * (1 + half) + half * want.abs() + 2.0 ** -25).all())
    assert bool((whole[:, cols:].float() == 7.0).all())


# ---- expert layer ----------------------------------------------------------------------------------------------------------------


def layer(g, experts, hidden, inter):
    def weights(n, k, *lead):
        w = torch.randn(*lead, n, k, generator=g, device="cuda") / math.sqrt(k)
        flat = [ref.quantize(m, E4, 128) for m in w.reshape(-1, n, k)]
        return (torch.stack([q for q, _ in flat]).float().to(E4).reshape(*lead, n, k),
                torch.stack([s for _, s in flat]).float().reshape(*lead, ref.nb(n), ref.nb(k)))

    return weights(inter, hidden, experts, 2) + weights(hidden, inter, experts)


def routes(g, tokens, experts, topk):
    ids = torch.rand(tokens, experts, generator=g, device="cuda").argsort(-1)[:, :topk].int().contiguous()
    w = torch.rand(tokens, topk, generator=g, device="cuda")
    return ids, w / w.sum(-1, keepdim=True)


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("tokens,experts,topk,hidden,inter", [(1, 4, 2, 128, 128), (1, 16, 4, 256, 400), (5, 8, 3, 272, 144), (20, 64, 6, 256, 128), (64, 4, 1, 512, 256),
                                                             (150, 8, 2, 384, 208), (700, 6, 3, 256, 272), (1000, 3, 2, 144, 640), (33, 1, 1, 1024, 16)])
def test_experts(lib, tokens, experts, topk, hidden, inter, xt):
    g = gen(tokens + hidden)
    w1, s1, w2, s2 = layer(g, experts, hidden, inter)
    ids, w = routes(g, tokens, experts, topk)
    if tokens > 4:
        ids[1] = -1             # padding: goes nowhere
        ids[2, 0] = experts     # no expert
        if topk > 1:
            ids[3, 1] = ids[3, 0]  # the same expert twice
    x = torch.randn(tokens, hidden + 16, generator=g, device="cuda").bfloat16().to(xt)[:, :hidden]
    whole, y = poison(tokens, hidden, xt, hidden + 8)
    ws = torch.full((lib.experts_workspace_bytes(hidden, inter, experts, topk, tokens, dtype={torch.float32: lib.F32, torch.float16: lib.F16, torch.bfloat16: lib.BF16}[xt]),),
                    0x7F, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        lib.fp8_experts(x, ids, w, w1, s1, w2, s2, y, ws)
    torch.cuda.synchronize()
    assert lib.fp8_status() == lib.OK
    want, err = ref.experts(x, ids, w, w1, s1, w2, s2, xt)
    off = (y.double() - want).abs()
    assert bool((off <= err).all()), float((off / err.clamp_min(1e-300)).max())
    assert bool((whole[:, hidden:].float() == 7.0).all())
    # on the whole: the output type's rounding twice, and few values of h that fell to the other side of a border
    assert float(off.norm()) <= (2 * torch.finfo(xt).eps + 2e-3) * float(want.norm())


def test_route_then_experts_and_its_parts(lib):
    """Router, sort, quantisation, products of groups and weighted sum in a row, and the expert layer on the same route."""
    g = gen(21)
    T, E, K, H, I = 90, 16, 4, 256, 256
    w1, s1, w2, s2 = layer(g, E, H, I)
    logits = torch.randn(T, E, generator=g, device="cuda")
    w, ids = run_route(lib, logits, K, kind="sigmoid", bias=torch.randn(E, generator=g, device="cuda") * 0.1)
    x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    y = torch.empty_like(x)
    ws = torch.empty(lib.experts_workspace_bytes(H, I, E, K, T), dtype=torch.uint8, device="cuda")
    lib.fp8_experts(x, ids, w, w1, s1, w2, s2, y, ws)
    want, err = ref.experts(x, ids, w, w1, s1, w2, s2, torch.bfloat16)
    assert bool(((y.double() - want).abs() <= err).all())

    offsets = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    rows, order = (torch.empty(T * K, dtype=torch.int32, device="cuda") for _ in range(2))
    lib.route_sort(ids, E, offsets, rows, order, torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))
    xs = x[order.long() // K]
    xq, xsc = torch.empty(T * K, H, device="cuda").to(E4), torch.empty(T * K, H // 128, device="cuda")
    lib.fp8_quantize(xs, xq, xsc)
    gate_up = torch.empty(T * K, 2 * I, device="cuda")
    lib.fp8_matmul(xq, xsc, w1.reshape(E, 2 * I, H), s1.reshape(E, 2 * I // 128, H // 128), gate_up, offsets=offsets)
    h = torch.nn.functional.silu(gate_up[:, :I]) * gate_up[:, I:]
    hq, hsc = torch.empty(T * K, I, device="cuda").to(E4), torch.empty(T * K, I // 128, device="cuda")
    lib.fp8_quantize(h, hq, hsc)
    parts = torch.empty(T * K, H, device="cuda", dtype=torch.bfloat16)
    lib.fp8_matmul(hq, hsc, w2, s2, parts, offsets=offsets)
    out = torch.empty_like(x)
    lib.route_combine(parts, rows.reshape(T, K), w, out)
    assert bool(((out.double() - want).abs() <= err).all())


@pytest.mark.parametrize("tokens", [3, 600])
def test_experts_graph(lib, tokens):
    """Two captured layers that share a workspace, replayed with other routes."""
    g = gen(22)
    E, K, H, I = 8, 2, 256, 128
    x = torch.randn(tokens, H, generator=g, device="cuda").bfloat16()
    ws = torch.empty(lib.experts_workspace_bytes(H, I, E, K, tokens), dtype=torch.uint8, device="cuda")
    ids, w = routes(g, tokens, E, K)
    nets = [layer(g, E, H, I) + (torch.empty_like(x),) for _ in range(2)]
    graphs = []
    for w1, s1, w2, s2, y in nets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.fp8_experts(x, ids, w, w1, s1, w2, s2, y, ws)
        graphs.append(graph)
    for seed in (1, 2):
        i2, w2_ = routes(gen(seed), tokens, E, K)
        ids.copy_(i2)
        w.copy_(w2_)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for w1, s1, w2, s2, y in nets:
            want, err = ref.experts(x, ids, w, w1, s1, w2, s2, torch.bfloat16)
            assert bool(((y.double() - want).abs() <= err).all())
    assert lib.fp8_status() == lib.OK
