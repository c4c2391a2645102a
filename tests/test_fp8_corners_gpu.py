"""8-bit float operators where their results hang on the numbers in between: slots that cancel, scores far below one, biases of both signs."""
import math

import pytest
import torch

import fp8_ref as ref

pytestmark = pytest.mark.gpu

E4 = torch.float8_e4m3fn
WIDE = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("tokens", [1, 20, 30, 100, 700])
def test_experts_slots_that_cancel(lib, tokens, xt):
    """Two slots of 784 * 257 and 784 * -256: in fewer than 14 bits their sum is another number, in 16-bit floats they are infinite.
    Everything is a whole number of few bits, so the result is exact up to the rounding of y."""
    H = I = 128
    x = torch.zeros(tokens, H, device="cuda")
    x[:, 0] = 448.0                                          # scale 1
    w1 = torch.zeros(2, 2, I, H, device="cuda")
    w1[:, :, :, 0] = 1.0
    s1 = torch.tensor([1.0, 2.0 ** -8], device="cuda").repeat(2).reshape(2, 2, 1, 1)  # gate 448, up 1.75: h = 784 = 448 * 1.75
    w2 = torch.zeros(2, H, I, device="cuda")
    n = torch.arange(H, device="cuda")
    w2[0, :, 0], w2[0, :, 1] = 256.0, 1.0
    w2[1, :, 0], w2[1, :, 1] = -256.0, (n % 8).float()
    s2 = torch.ones(2, 1, 1, device="cuda")
    ids = torch.tensor([0, 1], dtype=torch.int32, device="cuda").repeat(tokens, 1)
    ids[1::2] = ids[1::2].flip(1)
    w = torch.ones(tokens, 2, device="cuda") * 2.0 ** -(torch.arange(tokens, device="cuda") % 3)[:, None]
    y = torch.full((tokens, H), math.nan, device="cuda", dtype=xt)
    kind = {torch.float32: lib.F32, torch.float16: lib.F16, torch.bfloat16: lib.BF16}[xt]
    ws = torch.empty(lib.experts_workspace_bytes(H, I, 2, 2, tokens, dtype=kind), dtype=torch.uint8, device="cuda")
    lib.fp8_experts(x.to(xt), ids, w, w1.to(E4), s1, w2.to(E4), s2, y, ws)
    assert lib.fp8_status() == lib.OK
    want = 784.0 * (1.0 + (n % 8).float()) * w[:, :1]
    assert torch.equal(y, want.to(xt))


# ---- runs by the sum of their two largest choices ----------------------------------------------------------------------------------


def check_choice(lib, x, topk, kind, groups, topk_groups, bias=None):
    """Experts as in 64 bits, for every token."""
    w = torch.empty(x.shape[0], topk, device="cuda")
    ids = torch.full((x.shape[0], topk), -9, dtype=torch.int32, device="cuda")
    d = lib.make_route_desc(x.shape[1], topk, lib.SCORE_SOFTMAX if kind == "softmax" else lib.SCORE_SIGMOID, groups, topk_groups, lib.GROUP_TOP2)
    lib.route(d, x, w, ids, bias=bias)
    _, want = ref.route(x, topk, kind, groups, topk_groups, "top2", bias=bias)
    wrong = (ids.cpu() != want).any(-1).nonzero().flatten().tolist()
    assert not wrong, (len(wrong), wrong[0], ids[wrong[0]], want[wrong[0]])


RUNS = [(32, 16, 5), (64, 8, 4), (64, 32, 6), (60, 20, 4), (256, 8, 4), (256, 32, 4), (512, 16, 3), (1024, 32, 7)]


@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,topk_groups", RUNS)
def test_runs_of_small_scores(lib, experts, groups, topk_groups, kind, xt):
    """No bias, scores from e^-5 to e^-130: what 32 bits hold with few bits or not at all still decides between runs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(experts + groups)
    for below in (5.0, 20.0, 60.0, 80.0, 88.0, 95.0, 100.0, 103.0, 130.0):
        x = torch.randn(120, experts, generator=g, device="cuda") * 1.5 - below
        if kind == "softmax":
            x[:, 3] = 0.0
        check_choice(lib, x.to(xt), 3, kind, groups, topk_groups)


@pytest.mark.parametrize("kind,runs", [("sigmoid", [(-87.0, -88.5), (-87.4, -87.4)]), ("softmax", [(-103.9, -103.9), (-102.95, -200.0)])])
def test_two_runs_of_small_scores(lib, kind, runs):
    x = torch.full((1, 32), -300.0, device="cuda")
    x[0, 0] = 0.0 if kind == "softmax" else -300.0
    for i, pair in enumerate(runs):
        x[0, 8 * (i + 1):8 * (i + 1) + 2] = torch.tensor(pair)
    check_choice(lib, x, 2, kind, 4, 2 if kind == "softmax" else 1)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,topk_groups", RUNS)
def test_runs_with_large_biases_of_both_signs(lib, experts, groups, topk_groups, kind):
    """The two largest choices of a run cancel: their sum is of the size of the scores, its error of the size of the biases."""
    g = torch.Generator(device="cuda")
    g.manual_seed(experts)
    x = torch.randn(300, experts, generator=g, device="cuda") * 1.5
    size = experts // groups
    for large in (1e2, 1e3, 1e4, 1e6):
        bias = torch.full((groups, size), -large, device="cuda")
        bias[:, size // 2] = large
        check_choice(lib, x, 3, kind, groups, topk_groups, bias.reshape(-1).contiguous())
        # a few runs of that kind among others; sums of ordinary choices near to them
        bias[::3] = 0.01 * torch.randn(bias[::3].shape, generator=g, device="cuda")
        check_choice(lib, x, 3, kind, groups, topk_groups, bias.reshape(-1).contiguous())


@pytest.mark.parametrize("tokens", [1, 30, 150])
def test_experts_gates_far_below_zero(lib, tokens):
    """silu(v) = v / (1 + e^-v) of gates where 1 + e^-v does not fit into 32 bits or hardly does, with up values that bring h back.

    Gates, ups and the second product are exact, so what is left of the error is the logistic function's: the exponential to two units of its last
    place (steps of 2^-149 once it is subnormal), sum, quotient (two units) and two products; then amax / 448 and its product with 448."""
    num = torch.tensor([3 / 16, 25 / 128, 103 / 512, 27 / 128, 115 / 512, -27 / 128], dtype=torch.float64, device="cuda")
    E, H = num.numel(), 128
    gate = -448 * num                                        # -84, -87.5, -90.125, -94.5, -100.625, 94.5
    x = torch.zeros(E * tokens, H, device="cuda")
    x[:, 0] = 448.0                                          # scale 1
    w1 = torch.zeros(E, 2, H, H, device="cuda")
    w1[:, 0, :, 0], w1[:, 1, :, 0] = -1.0, 1.0
    s1 = torch.ones(E, 2, 1, 1, device="cuda")
    s1[:, 0, 0, 0] = num.float()
    s1[:5, 1] = 2.0 ** 90
    w2 = torch.zeros(E, H, H, device="cuda")
    w2[:, :, 5] = 1.0
    ids = (torch.arange(E * tokens, dtype=torch.int32, device="cuda") % E)[:, None].contiguous()
    w = torch.ones(E * tokens, 1, device="cuda")
    y = torch.full((E * tokens, H), math.nan, device="cuda")
    ws = torch.empty(lib.experts_workspace_bytes(H, H, E, 1, E * tokens, dtype=lib.F32), dtype=torch.uint8, device="cuda")
    lib.fp8_experts(x, ids, w, w1.to(E4), s1, w2.to(E4), torch.ones(E, 1, 1, device="cuda"), y, ws)
    assert lib.fp8_status() == lib.OK
    want = gate / (1 + torch.exp(-gate)) * 448 * s1[:, 1, 0, 0].double()
    error = 2 * torch.where(gate < 0, 2.0 ** -149 / torch.exp(gate), 0.0) + 12 * 2.0 ** -23
    e = ids[:, 0].long()
    assert bool(((y.double() - want[e][:, None]).abs() <= (error * want.abs())[e][:, None]).all()), (y[:E, 0], want)


# ---- failure detection -------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("form,rows", [(0, 5), (1, 600)])
def test_bounded_wait_reports_timeout_and_products_stay_usable(lib, form, rows):
    """A wait that cannot complete ends by itself, is reported once, and the kernels run on."""
    lib.selftest_fp8_wait(form)
    assert lib.fp8_status() == lib.E_TIMEOUT
    assert lib.fp8_status() == lib.OK
    a = torch.randint(-3, 4, (rows, 256), device="cuda").float()
    b = torch.randint(-3, 4, (200, 256), device="cuda").float()
    y = torch.empty(rows, 200, device="cuda")
    lib.fp8_matmul(a.to(E4), torch.ones(rows, 2, device="cuda"), b.to(E4), torch.ones(2, 2, device="cuda"), y)
    assert torch.equal(y, a @ b.t()) and lib.fp8_status() == lib.OK


# ---- weights -----------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("experts", [512, 600, 1000, 1024])
def test_weights_of_a_flat_softmax(lib, experts):
    """Very many scores of about the same size: every one of them may add a rounding to the sum that the weights are divided by.  Tolerance: eight
    units of 2^-24, as for all weights; two each for the exponentials in the sum and the weight's own, one each for the sum's and the quotient's
    rounding to 32 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(experts)
    d = lib.make_route_desc(experts, 8, lib.SCORE_SOFTMAX, renormalise=False)
    for below in torch.linspace(0.0, 16.0, 33).tolist():
        x = torch.randn(2000, experts, generator=g, device="cuda") * 0.001 - below
        x[:, 7] = 0.0
        w = torch.empty(2000, 8, device="cuda")
        ids = torch.empty(2000, 8, dtype=torch.int32, device="cuda")
        lib.route(d, x, w, ids)
        want = torch.softmax(x.double(), -1).gather(1, ids.long())
        off = (w.double() - want).abs() / want
        assert float(off.max()) <= 8 * 2.0 ** -24, (below, float(off.max()) * 2 ** 24)
