"""4-bit float operators on the device, at the corners that their other tests leave out, against the definitions in 64 bits (fp4_ref)."""
import pytest
import torch

import fp4_ref as ref
from fp4_ref import MX, NV
from test_fp4_gpu import check_experts, layer, routes, run_experts

FMT = pytest.mark.parametrize("fmt", [MX, NV], ids=["mx", "nv"])
U = 2.0 ** -24  # half a step of fp32 at most, relative

pytestmark = pytest.mark.gpu


def code_of(lib, call, *args, **kw):
    with pytest.raises(lib.B2CError) as e:
        call(*args, **kw)
    return e.value.code


def test_empty_matrices_are_refused(lib):
    """A stack of matrices without rows, a layer without an inner or a hidden size, all on the device."""
    q, s = lib.fp4_empty(3, 64, lib.NVFP4)
    b, bs = lib.fp4_empty((4, 0), 64, lib.NVFP4)
    offsets = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert code_of(lib, lib.fp4_matmul, q, s, b, bs, torch.zeros(3, 0, device="cuda"), offsets=offsets) == lib.E_INVALID_ARG
    ids, weights, ws = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, 1, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    for hidden, inter in ((64, 0), (0, 64)):
        (w1, s1), (w2, s2) = lib.fp4_empty((2, 2, inter), hidden, lib.NVFP4), lib.fp4_empty((2, hidden), inter, lib.NVFP4)
        x, y = (torch.zeros(3, hidden, device="cuda") for _ in range(2))
        assert code_of(lib, lib.fp4_experts, x, ids, weights, w1, s1, w2, s2, y, ws) == lib.E_INVALID_ARG


# ---- quantisation ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("g", [1.1 * 2.0 ** -100, 1.9999999 * 2.0 ** -100, 2.0 ** -100, 1.3333334 * 2.0 ** -97, 1.7 * 2.0 ** -88, 0.77, 1.1 * 2.0 ** 99, 2.0 ** 100])
def test_quantize_next_to_borders_of_any_factor(lib, g):
    """fp32 numbers within a few units of the borders between values, and blocks whose largest is within a few of those between scales, for the smallest
    and the largest factors and scales: equal to the quotients in 64 bits in every value."""
    f = torch.tensor([g], dtype=torch.float32, device="cuda")
    g = float(f)
    v = torch.tensor(ref.VALUES, dtype=torch.float64)
    mid = (v[:-1] + v[1:]) / 2
    scales = ref.scale_numbers(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn), NV)
    near = lambda a, d: (a.float().view(torch.int32) + d).view(torch.float32)  # noqa: E731
    rows = []
    for s in scales[1:].tolist():
        for d in range(-3, 4):
            x = near(mid * s * g, d)
            rows.append(torch.cat([x, -x, torch.tensor([6 * s * g, 0.0]).float()]))
    borders = (scales[:-1] + scales[1:]) / 2
    for d in range(-3, 4):
        x = torch.zeros(126, 16)
        x[torch.arange(126), torch.arange(126) % 16] = near(borders * 6 * g, d) * (-1) ** d
        rows += list(x)
    x = torch.stack(rows).cuda()
    q, s = torch.empty(x.shape[0], 8, dtype=torch.uint8, device="cuda"), torch.empty(x.shape[0], 1, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    lib.fp4_quantize(x, q, s, global_scale=f)
    want, scale = ref.quantize(x, NV, f)
    assert bool((ref.scale_numbers(s, NV) == scale).all()) and bool((ref.unpack(q, 16) == want).all())


# ---- hidden rows of an expert layer, seen through a second matrix that is the identity ---------------------------------------------------

def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def identity(lib, experts, n, fmt):
    """[experts, n, n] in 4 bits: the layer's result for a token of one expert with weight 1 is its hidden row as quantised (times the factor)."""
    code = 2 * torch.eye(n, dtype=torch.uint8, device="cuda")  # (code 2 is 1.0)
    q, s = lib.fp4_empty((experts, n), n, fmt)
    q.copy_(ref.pack(code).expand(experts, n, n // 2))
    s.view(torch.uint8).fill_(127 if fmt == MX else 56)
    return q, s


def run_layer(lib, x, ids, w1, s1, w2, s2, fmt, **factors):
    T, H = x.shape
    n = lib.fp4_experts_workspace_bytes(H, w1.shape[2], w1.shape[0], ids.shape[1], T, fmt, lib.F32)
    y = torch.full_like(x, 9.0)
    lib.fp4_experts(x, ids, torch.ones(ids.shape, device="cuda"), w1, s1, w2, s2, y, torch.empty(n, dtype=torch.uint8, device="cuda"), **factors)
    assert lib.fp4_status() == lib.OK
    return y


def block_max(v):
    return v.reshape(v.shape[0], -1, 32).amax(-1)


# (one expert: up to 4 tokens go to the two kernels for few, tiles of 16 rows, tiles of 128)
@pytest.mark.parametrize("T", [2, 4, 10, 100])
def test_gates_far_below_zero(lib, T):
    """Gates from -6 to -153 (a few below it) beside up values of up to 2^115: e^gate leaves the range of fp32, the gated product and its scale do not.  Sums of the first
    product are whole multiples of a power of two below 2^24 of it, so they are exact."""
    n, g = 512, gen(T)
    codes = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda")  # noqa: E731
    x = torch.zeros(T, n, device="cuda")
    x[:, :32] = torch.tensor(ref.VALUES, device="cuda")[codes(1, 8, T, 32)]
    x[:, 31] = 6.0  # (the scale is 1)
    w, sw = lib.fp4_empty((1, 2, n), n, MX)
    full = torch.zeros(2, n, n, dtype=torch.long, device="cuda")
    # a block's 32 columns have the same weights but for the first: their gates are near each other, so that many of a block are not rounded to zero
    full[:, :, :32] = codes(1, 5, 2, n // 32, 32).repeat_interleave(32, 1)
    full[:, :, 0] = codes(1, 6, 2, n)
    full[0, :, :32] += 8  # (gates are negative)
    w[0] = ref.pack(full)
    shift = torch.zeros(2, n // 32, dtype=torch.long, device="cuda")
    shift[0] = torch.tensor([0, 0, 0, 0, 0, -1, 0, 0, -4, 0, 0, 0, 0, -2, 0, 0], device="cuda")
    shift[1] = torch.tensor([108, 104, 100, 96, 92, 40, 84, 106, 3, 100, 90, 95, 105, 20, 70, 108], device="cuda")
    sw.view(torch.uint8)[0] = (127 + shift).repeat_interleave(32, 1)[:, :, None].to(torch.uint8)
    y = run_layer(lib, x, torch.zeros(T, 1, dtype=torch.int32, device="cuda"), w, sw, *identity(lib, 1, n, MX), MX).double()

    gate, up = (x.double() @ ref.values(w[0, j], sw[0, j], MX).t() for j in (0, 1))
    assert float(gate.max()) > -20 and float((gate < -88).double().mean()) > 0.5
    h = gate / (1 + torch.exp(-gate)) * up
    # in units of U: the power of two 4 (2^-22), its exponent's rounding and constant 1.25 |gate|, the sum 1, its reciprocal 2, three products
    dh = (10 + 1.25 * gate.abs()) * U * h.abs()
    amax = ref.block_amax(h, MX)
    scale = ref.scales_of(amax, MX)
    damax = ref.block_amax(dh, MX)
    low, high = (ref.rounded(h.abs() + d * dh, scale, MX) * ref.spread(scale, n, MX) for d in (-1, 1))
    sure = (ref.scales_of(amax - damax, MX) == scale) & (ref.scales_of(amax + damax, MX) == scale) & (amax > 2.0 ** -118)  # (results below are not normal)
    sure = ref.spread(sure & (block_max(gate) > -153), n, MX) & (gate > -153) & (low == high)  # (h is 0 below)
    assert float(sure.double().mean()) > 0.5 and float((sure & (low > 0) & (gate < -88)).double().mean()) > 0.1
    assert bool((y == -low)[sure].all())


# (a row an expert goes to the two kernels for few tokens, 8 and 30 to tiles of 16 and 64 rows, 64 to those of 128)
@pytest.mark.parametrize("rows", [1, 8, 30, 64])
def test_hidden_rows_next_to_borders(lib, rows):
    """Hidden rows within some units of 2^-24 of the borders between two 4-bit values: who is further than 3 units from one is on its right side.
    A token's only value is 6, gates are so large that silu is the gate itself, and 36 times the square of an expert's factor is next to h's, so the
    columns of a block are 6 and the seven borders times the scale that the gate's weights have, nearly; everything before h is exact but for its
    three roundings, which are made here too."""
    E, n, g = 32, 64, gen(rows)
    up = torch.tensor([6.0] + 2 * [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] + [5.0], dtype=torch.float64, device="cuda").repeat(n // 16)
    x = torch.zeros(E, n, device="cuda")
    x[:, 0] = 6.0
    moved = torch.linspace(-6, 6, E, dtype=torch.float64, device="cuda") * U
    # factors whose reciprocal by way of six times them and back, each step rounded, is furthest off (up to three units)
    some = (torch.rand(1 << 20, generator=g, device="cuda") + 1) * 4096
    worst = (6.0 * (1.0 / (6.0 * some)).double() * some.double() - 1).abs().topk(24).indices
    for gh in some[worst][:, None]:
        f1 = (gh.double() / 36 * (1 + moved)).sqrt().float()
        code = torch.randint(56, 120, (E, n // 16), generator=g, device="cuda", dtype=torch.uint8).repeat_interleave(16, 1)  # scales from 1 to 240
        w, sw = lib.fp4_empty((E, 2, n), n, NV)
        w.zero_()
        w[..., 0] = 2  # 1.0 in the first column, times the block's scale
        sw.view(torch.uint8)[:, 0, :, 0] = code
        sw[:, 1, :, 0] = up.float().to(torch.float8_e4m3fn)
        ids = torch.arange(E, dtype=torch.int32, device="cuda").repeat(rows)[:, None]
        y = run_layer(lib, x.repeat(rows, 1), ids, w, sw, *identity(lib, E, n, NV), NV, w1_global=f1, h_global=gh)

        scale = ref.scale_numbers(code, NV)
        gate = (6 * scale).float() * f1[:, None]
        h = (gate * ((6 * up).float() * f1[:, None])).double()  # (two products rounded, and theirs)
        assert float(gate.min()) >= 40  # (e^-40 does not count beside 1)
        off = h / (up * scale * gh.double()) - 1
        assert bool((off.abs() < 12 * U).all()) and float((off.abs() > 3 * U).double().mean()) > 0.2
        ends = [(ref.round4(h * (1 + d * 3 * U) / (scale * gh.double())) * scale).float() * gh for d in (-1, 1)]
        y = y.reshape(rows, E, n)
        wrong = (y != ends[0]) & (y != ends[1])
        assert not bool(wrong.any()), (int(wrong.sum()), float(off[wrong.any(0)].abs().max() / U))


# ---- expert layers of real sizes -------------------------------------------------------------------------------------------------------

# Reductions of more than one group of scales (1024) and of more stages (256 each) than any ring holds, last stages that are not full, in both products.
# One and 16 tokens and 100 of many experts go to the two kernels for few, the others to tiles of 32, 64 and 128 rows.
@FMT
@pytest.mark.parametrize("T,experts,topk,hidden,inter", [(1, 16, 8, 2336, 1312), (16, 16, 4, 1312, 2336), (3, 4, 4, 2336, 2336), (100, 32, 1, 1056, 2080), (100, 16, 3, 2336, 1312),
                                                         (100, 8, 3, 1312, 2336), (150, 3, 2, 2336, 1312), (400, 6, 3, 1312, 2336)])
def test_experts_long_reductions(lib, T, experts, topk, hidden, inter, fmt):
    w = layer(lib, hidden, inter, experts, fmt, T)
    x = torch.randn(T, hidden, generator=gen(T + 1), device="cuda").bfloat16()
    ids, weights = routes(T, experts, topk, T + 2)
    gx, gh = (torch.tensor([v / 2688], device="cuda") for v in (6, 9)) if fmt == NV else (None, None)
    y = run_experts(lib, x, ids, weights, w, fmt, gx, gh, extra=64)
    check_experts(y, x, ids, weights, w, fmt, gx, gh)


# Routes on which the average says little: one expert has 15 to 33 of a few tokens (more than one tile of the kernels for few), or most of many.
@FMT
@pytest.mark.parametrize("T,experts,topk,most", [(64, 64, 4, 15), (64, 64, 4, 16), (64, 64, 4, 17), (64, 64, 4, 32), (64, 64, 4, 33), (64, 64, 4, 64), (40, 128, 8, 40),
                                                 (600, 64, 2, 600), (700, 40, 4, 650)])
def test_experts_skewed_routes(lib, T, experts, topk, most, fmt):
    hidden, inter, hot = 288, 160, 5
    w = layer(lib, hidden, inter, experts, fmt, most)
    x = torch.randn(T, hidden, generator=gen(most + 1), device="cuda").half()
    ids, weights = routes(T, experts - 1, topk, most + 2)
    ids += ids >= hot  # (all but the hot one)
    chosen = torch.randperm(T, generator=gen(most + 3), device="cuda")[:most]
    ids[chosen, chosen % topk] = hot
    assert int((ids == hot).sum()) == most
    y = run_experts(lib, x, ids, weights, w, fmt, extra=64)
    check_experts(y, x, ids, weights, w, fmt)


@FMT
@pytest.mark.parametrize("T,experts", [(2, 16), (30, 64), (200, 16)])
def test_experts_many_slots(lib, T, experts, fmt):
    """Eight slots a token, of which every third token has two."""
    w = layer(lib, 512, 256, experts, fmt, T)
    x = torch.randn(T, 512, generator=gen(T + 1), device="cuda").bfloat16()
    ids, weights = routes(T, experts, 8, T + 2)
    ids[1::3, 2:] = -1
    y = run_experts(lib, x, ids, weights, w, fmt)
    check_experts(y, x, ids, weights, w, fmt)
